// The recurrence with a matrix state, S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, on the CUDA cores: float32
// arithmetic throughout, any head dimension up to 256, any stride and alignment.  Also the kernels that finish a
// backward pass and the one-token step.
//
// One "pass" serves the forward direction and all three gradients.  With c_i the running sum of the log decays inside a
// chunk, X, Y, Z the three tensors in the roles of query, key and value:
//     forward :  out_i = scale * ( sum_{j<=i} e^{c_i-c_j} (X_i.Y_j) Z_j + e^{c_i} X_i S ),   S' = e^{c_C} S + sum_j e^{c_C-c_j} Y_j Z_j^T
//     reversed:  out_j = scale * ( sum_{i>=j} e^{c_i-c_j} (X_j.Y_i) Z_i + e^{c_C-c_j} X_j S ), S' = e^{c_C} S + sum_i e^{c_i} Y_i Z_i^T
// o = forward(q, k, v); dq = forward(dO, v, k) from S0^T; dk = reversed(v, dO, q) from (dS_T)^T; dv = reversed(k, q, dO)
// from dS_T, which ends at dS_0.  Differentiating the formula for o gives each line at once: e^{c_i-c_j} is common to all.
// Every exponent is <= 0 for decays <= 1, so nothing overflows whatever the length.
//
// The log decays: with W_ij = scale e^{c_i-c_j} (q_i.k_j)(dO_i.v_j), dlog_a_t = sum over all pairs i >= t > j of W_ij, plus
// what crosses t from S_0 and to dS_T.  (It is also the reverse running sum of q.dq - k.dk, but there the pairs on one side
// of t cancel, and where decays are strong nothing else is left.)  Sorted by where i and j lie beside t's chunk, with S the
// state before the chunk and D the gradient of the state after it:
//     both in the chunk          sum_{i>=t>j} W_ij
//     j before, i in it          sum_{i>=t} scale e^{c_i} q_i^T S dO_i
//     j in it, i behind          sum_{j<t} e^{c_C-c_j} k_j^T D v_j
//     j before, i behind         e^{c_C} <S, D>
// No term cancels another.  The two passes leave S and D of every chunk behind for it.
#pragma once
#include "ha_common.cuh"

namespace ha {

constexpr int kSimtChunk = 32;   // tokens of a chunk
constexpr int kSimtThreads = 256;

struct Pass {
    Rows x, y, z;
    const float* log_a;
    long long ab, at, ah;
    const int* lengths;
    int batch, tokens, heads, dx, dz;
    float scale;
    const float* s_in;   // [batch, heads, dx, dz], or [.., dz, dx] where s_in_t
    float* s_out;        // [batch, heads, dx, dz]
    int s_in_t;
    float s_in_mul, s_out_mul;
    void* out;           // [batch, tokens, heads, dz] through its strides
    long long ob, ot, oh;
    float* dump;         // [batch * heads, chunks, dx, dz]: the state before each chunk, or NULL
    // A sequence cut into segments of seg_chunks chunks: each starts from seg_state[bh][segment] ([dx, dz])
    int segments, seg_chunks;
    float* seg_state;
    float* seg_decay;
    int rev;
    Fault* fault;
    unsigned long long call_id;
};
// Passes over the same sequences that do not depend on one another go in one launch, blockIdx.y each.
struct Passes {
    Pass p[3];
};

// Columns c0 + lane + 32 u (u < kN) of a warp's four of the rows t0 .. t0 + 31, zeros where there is nothing; and their way to
// shared memory.
template <int kN, class T>
__device__ __forceinline__ void load_rows(float (&v)[4 * kN], const T* from, long long st, int c0, int dim, int t0, int live) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int u = 0; u < kN; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + warp + 8 * i, c = c0 + lane + 32 * u;
            v[4 * u + i] = t < live && c < dim ? to_f(from[t * st + c]) : 0.0f;
        }
}
template <int kN>
__device__ __forceinline__ void keep_rows(const float (&v)[4 * kN], float* to, int pitch, int c0, int width) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int u = 0; u < kN; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + lane + 32 * u < width) to[(warp + 8 * i) * pitch + c0 + lane + 32 * u] = v[4 * u + i];
}
__device__ __forceinline__ void add4(float4& acc, float w, const float4& v) {
    acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
}

// A CTA has kCols columns of Z and of the state and walks the chunks of its segment.  The products read shared memory more than
// they compute: a 16-byte read of a warp costs it four turns, whatever is read twice.  So a thread has four columns of kPer
// output rows and of four state rows, which share those reads (24 sequences of up to 1000 tokens, dimension 64: 69 us with one
// row for 32 columns, 43 us with two for 64; the sums of the states before it 25 us and 16 us).  The next chunk's first 64
// columns travel meanwhile: waiting for them took half of a chunk's time.  With an output a thread spills 52 to 68 bytes at the 128
// registers that two CTAs leave it.
template <class T, bool kRev, class OutT, bool kStateOnly, int kCols>
__device__ __forceinline__ void simt_pass(const Pass& p) {
    constexpr int kLanes = kCols / 4, kSweep = kSimtThreads / kLanes, kPer = kSimtChunk / kSweep;
    extern __shared__ __align__(16) float sm[];
    const int dxp = p.dx + 4 - (p.dx & 3) + ((p.dx & 3) ? 4 : 0);  // a multiple of 4, at least dx + 4: rows shifted by 4 banks
    float* xs = sm;                                  // [32][dxp]
    float* ys = xs + kSimtChunk * dxp;               // [32][dxp]
    float* zs = ys + kSimtChunk * dxp;               // [32][kCols]
    float* zw = zs + kSimtChunk * kCols;         // [32][kCols] times the state's weight
    float* st = zw + kSimtChunk * kCols;         // [dx][kCols]
    float* pr = st + p.dx * kCols;               // [32][33]
    __shared__ float c_hi[kSimtChunk], c_lo[kSimtChunk], w_in[kSimtChunk], w_st[kSimtChunk];
    __shared__ float s_whole;

    const int tid = threadIdx.x, ztiles = (p.dz + kCols - 1) / kCols;
    const int cuts = kStateOnly ? p.segments - 1 : p.segments;  // the last segment's own state is not needed by another
    const int segment = blockIdx.x % cuts, item = blockIdx.x / cuts;
    const int z0 = item % ztiles * kCols;
    const int bh = item / ztiles, b = bh / p.heads, h = bh % p.heads;
    if (bh >= p.batch * p.heads) return;  // another pass has more columns
    const int live = live_tokens(p.lengths, b, p.tokens);
    const T* gx = static_cast<const T*>(p.x.ptr) + b * p.x.sb + (h / p.x.div) * p.x.sh;
    const T* gy = static_cast<const T*>(p.y.ptr) + b * p.y.sb + (h / p.y.div) * p.y.sh;
    const T* gz = static_cast<const T*>(p.z.ptr) + b * p.z.sb + (h / p.z.div) * p.z.sh;
    const float* ga = p.log_a + b * p.ab + h * p.ah;
    OutT* go = static_cast<OutT*>(p.out) + b * p.ob + h * p.oh;

    const long long plane = (long long)bh * p.dx * p.dz;
    float* const seg = p.segments > 1 ? p.seg_state + ((long long)bh * p.segments + segment) * p.dx * p.dz : nullptr;
    for (int e = tid; e < p.dx * kCols; e += kSimtThreads) {
        const int k = e / kCols, z = z0 + e % kCols;
        float v = 0.0f;
        if (!kStateOnly && z < p.dz) {
            if (seg) v = seg[(long long)k * p.dz + z];
            else if (p.s_in) v = p.s_in[plane + (p.s_in_t ? (long long)z * p.dx + k : (long long)k * p.dz + z)] * p.s_in_mul;
        }
        st[e] = v;
    }
    const int chunks = (p.tokens + kSimtChunk - 1) / kSimtChunk;
    const int first = min(chunks, segment * p.seg_chunks), last = min(chunks, first + p.seg_chunks);
    double total = 0.0;
    // the next chunk's first 64 columns, on their way while this one is worked on
    float x_next[8], y_next[8], z_next[kCols / 8], a_next = 0.0f;
    auto fetch = [&](int n) {
        if (n >= last) return;
        const int t0 = (kRev ? chunks - 1 - n : n) * kSimtChunk;
        if (!kStateOnly) load_rows<2>(x_next, gx, p.x.st, 0, p.dx, t0, live);
        load_rows<2>(y_next, gy, p.y.st, 0, p.dx, t0, live);
        load_rows<kCols / 32>(z_next, gz, p.z.st, z0, p.dz, t0, live);
        a_next = tid < 32 && t0 + tid < live ? ga[(t0 + tid) * p.at] : 0.0f;
    };
    bool fetched = false;
    for (int n = first; n < last; ++n) {
        const int t0 = (kRev ? chunks - 1 - n : n) * kSimtChunk;
        if (t0 >= live && !p.dump) {  // nothing in it: the state passes as it is
            if (!kStateOnly)
                for (int e = tid; e < kSimtChunk * kCols; e += kSimtThreads) {
                    const int t = t0 + e / kCols, z = z0 + e % kCols;
                    if (t < p.tokens && z < p.dz) go[t * p.ot + z] = from_f<OutT>(0.0f);
                }
            continue;
        }
        if (!fetched) fetch(n);
        fetched = true;
        __syncthreads();
        if (!kStateOnly && p.dump)
            for (int e = tid; e < p.dx * kCols; e += kSimtThreads) {
                const int k = e / kCols, z = z0 + e % kCols;
                if (z < p.dz) p.dump[(((long long)bh * chunks + t0 / kSimtChunk) * p.dx + k) * p.dz + z] = st[e];
            }
        if (!kStateOnly) keep_rows<2>(x_next, xs, dxp, 0, dxp);
        keep_rows<2>(y_next, ys, dxp, 0, dxp);
        keep_rows<kCols / 32>(z_next, zs, kCols, 0, kCols);
        for (int c0 = 64; c0 < dxp; c0 += 64) {
            float x[8], y[8];
            if (!kStateOnly) load_rows<2>(x, gx, p.x.st, c0, p.dx, t0, live);
            load_rows<2>(y, gy, p.y.st, c0, p.dx, t0, live);
            if (!kStateOnly) keep_rows<2>(x, xs, dxp, c0, dxp);
            keep_rows<2>(y, ys, dxp, c0, dxp);
        }
        if (tid < 32) {
            // running sums of the log2 decays, in 64 bits and handed on as two floats: a reset (-10000) must not cost the
            // differences of the sums after it their low bits
            const float a = a_next < kReset ? kReset : a_next;
            double c = (double)a * 1.4426950408889634;
            for (int o = 1; o < 32; o *= 2) {
                const double u = __shfl_up_sync(~0u, c, o);
                if (tid >= o) c += u;
            }
            const double whole = __shfl_sync(~0u, c, 31);
            total += whole;
            c_hi[tid] = (float)c;
            c_lo[tid] = (float)(c - (double)(float)c);
            w_in[tid] = ex2((float)(kRev ? whole - c : c));
            w_st[tid] = ex2((float)(kRev ? c : whole - c));
            if (tid == 31) s_whole = ex2((float)whole);
        }
        fetch(n + 1);
        __syncthreads();
        if (!kStateOnly) {  // P, four columns of one row each
            const int i = tid >> 3, j0 = tid & 7;
            float acc[4] = {};
#pragma unroll 4
            for (int k = 0; k < dxp - 4; k += 4) {
                const float4 a = *reinterpret_cast<const float4*>(xs + i * dxp + k);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float4 c = *reinterpret_cast<const float4*>(ys + (j0 + 8 * m) * dxp + k);
                    acc[m] = fmaf(a.x, c.x, fmaf(a.y, c.y, fmaf(a.z, c.z, fmaf(a.w, c.w, acc[m]))));
                }
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int j = j0 + 8 * m, late = kRev ? j : i, early = kRev ? i : j;
                const float d = (c_hi[late] - c_hi[early]) + (c_lo[late] - c_lo[early]);
                pr[i * 33 + j] = early <= late ? acc[m] * ex2(d) : 0.0f;
            }
        }
        for (int e = tid; e < kSimtChunk * kCols; e += kSimtThreads) zw[e] = zs[e] * w_st[e / kCols];
        __syncthreads();
        const int z = tid % kLanes * 4, r0 = tid / kLanes;
        if (!kStateOnly) {  // four columns of kPer output rows each
            float4 in[kPer] = {}, far[kPer] = {};
#pragma unroll 8
            for (int j = 0; j < kSimtChunk; ++j) {
                const float4 v = *reinterpret_cast<const float4*>(zs + j * kCols + z);
#pragma unroll
                for (int u = 0; u < kPer; ++u) add4(in[u], pr[(r0 + u * kSweep) * 33 + j], v);
            }
#pragma unroll 8
            for (int k = 0; k < p.dx; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(st + k * kCols + z);
#pragma unroll
                for (int u = 0; u < kPer; ++u) add4(far[u], xs[(r0 + u * kSweep) * dxp + k], v);
            }
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int i = r0 + u * kSweep;
                const float in4[4] = {in[u].x, in[u].y, in[u].z, in[u].w}, far4[4] = {far[u].x, far[u].y, far[u].z, far[u].w};
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    if (t0 + i < p.tokens && z0 + z + m < p.dz)
                        go[(t0 + i) * p.ot + z0 + z + m] =
                            from_f<OutT>(t0 + i < live ? p.scale * (in4[m] + decayed(w_in[i], far4[m])) : 0.0f);
            }
            __syncthreads();
        }
        for (int k0 = r0; k0 < p.dx; k0 += 4 * kSweep) {  // the state, four rows at a time
            float4 acc[4] = {};
#pragma unroll 4
            for (int j = 0; j < kSimtChunk; ++j) {
                const float4 v = *reinterpret_cast<const float4*>(zw + j * kCols + z);
#pragma unroll
                for (int u = 0; u < 4; ++u) add4(acc[u], ys[j * dxp + min(k0 + u * kSweep, p.dx)], v);  // column dx is there, and zero
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k0 + u * kSweep < p.dx) {
                    float4* own = reinterpret_cast<float4*>(st + (k0 + u * kSweep) * kCols + z);
                    const float4 s = *own;
                    *own = make_float4(acc[u].x + decayed(s_whole, s.x), acc[u].y + decayed(s_whole, s.y), acc[u].z + decayed(s_whole, s.z),
                                       acc[u].w + decayed(s_whole, s.w));
                }
        }
    }
    __syncthreads();
    if (kStateOnly) {
        for (int e = tid; e < p.dx * kCols; e += kSimtThreads) {
            const int k = e / kCols, z = z0 + e % kCols;
            if (z < p.dz) seg[(long long)k * p.dz + z] = st[e];
        }
        if (tid == 0 && z0 == 0) p.seg_decay[bh * p.segments + segment] = ex2((float)total);
    } else if (p.s_out && segment == p.segments - 1) {
        for (int e = tid; e < p.dx * kCols; e += kSimtThreads) {
            const int k = e / kCols, z = z0 + e % kCols;
            if (z < p.dz) p.s_out[plane + (long long)k * p.dz + z] = st[e] * p.s_out_mul;
        }
    }
}
// Both directions in one kernel: one register count, but no decision inside the loops (a direction read at run time took 6%).
template <class T, class OutT, bool kStateOnly, int kCols>
__global__ void __launch_bounds__(kSimtThreads, 2) simt_pass_kernel(const __grid_constant__ Passes passes) {
    const Pass& p = passes.p[blockIdx.y];
    // nothing here waits, but the header of a kept workspace may still show what an earlier call met
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.fault->started_id = p.call_id;
    if (p.rev) simt_pass<T, true, OutT, kStateOnly, kCols>(p);
    else simt_pass<T, false, OutT, kStateOnly, kCols>(p);
}
inline size_t simt_pass_smem(int dx, int cols) {
    const int dxp = dx + 4 - (dx & 3) + ((dx & 3) ? 4 : 0);
    return sizeof(float) * (size_t)(2 * kSimtChunk * dxp + 2 * kSimtChunk * cols + dx * cols + kSimtChunk * 33);
}

// What each segment starts from: the states that the segments would end at from zero (left by the state-only pass in
// seg_state) joined in order.  A thread has one element and loads eight segments' before it stores one: the chain itself is
// one multiply-add a segment, memory's latency was all of the 16 us that one load at a time took (18 segments of 8 heads).
template <class P>
__device__ __forceinline__ void join_segments(const P& p) {
    const int plane = p.dx * p.dz, tiles = (plane + 255) / 256;
    const int bh = blockIdx.x / tiles, e = blockIdx.x % tiles * 256 + threadIdx.x;
    if (e >= plane) return;
    const int k = e / p.dz, z = e % p.dz, last = p.segments - 1;
    const float* decay = p.seg_decay + (long long)bh * p.segments;
    float* at = p.seg_state + (long long)bh * p.segments * plane + e;
    float cur = p.s_in ? p.s_in[(long long)bh * plane + (p.s_in_t ? z * p.dx + k : e)] * p.s_in_mul : 0.0f;
    constexpr int kAhead = 8;
    for (int s0 = 0; s0 <= last; s0 += kAhead) {
        float own[kAhead], d[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            own[i] = s0 + i < last ? at[(long long)(s0 + i) * plane] : 0.0f;
            d[i] = s0 + i < last ? decay[s0 + i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s0 + i <= last) {
                at[(long long)(s0 + i) * plane] = cur;
                cur = decayed(d[i], cur) + own[i];
            }
    }
}
template <class P>
__global__ void __launch_bounds__(256) join_segments_kernel(const __grid_constant__ P p) { join_segments(p); }
__global__ void __launch_bounds__(256) join_passes_kernel(const __grid_constant__ Passes passes) { join_segments(passes.p[blockIdx.y]); }

// dst[b, t, g, :] = the sum over the heads that read head g, rounded once; zero behind a sequence's end.
template <class T>
__global__ void sum_heads_kernel(const float* src, T* dst, const int* lengths, int tokens, int heads, int groups, int dim,
                                 long long total) {
    const int share = heads / groups;
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long long)gridDim.x * blockDim.x) {
        const int d = (int)(e % dim);
        const long long row = e / dim;  // (b, t, g)
        const int g = (int)(row % groups);
        const long long bt = row / groups;
        float s = 0.0f;
        if ((int)(bt % tokens) < live_tokens(lengths, (int)(bt / tokens), tokens)) {
            const float* from = src + (bt * heads + (long long)g * share) * dim + d;
            for (int i = 0; i < share; ++i) s += from[(long long)i * dim];
        }
        dst[e] = from_f<T>(s);
    }
}

// dlog_a of one chunk of one (batch, head) from the definition above.  `before` and `behind` are what the dq pass and the dk
// pass left: S^T and D^T / scale of every chunk, [dv, dk].  part (fixed decays): only the sum over the chunk's tokens.
struct DecayGrad {
    Rows q, k, v, g;
    const float* log_a;
    long long ab, at, ah;
    const int* lengths;
    int tokens, heads, chunks, dk, dv;
    float scale;
    const float *before, *behind;
    float* dlog_a;
    double* part;
};
constexpr int kDecayThreads = 256;

template <class T>
__global__ void __launch_bounds__(kDecayThreads) decay_grad_kernel(const DecayGrad p) {
    extern __shared__ float sm[];
    // token-minor copies: one 16-byte load has four tokens of one element
    float* qs = sm;                                  // [dk][32]
    float* ks = qs + p.dk * kSimtChunk;              // [dk][32]
    float* vs = ks + p.dk * kSimtChunk;              // [dv][32]
    float* gs = vs + p.dv * kSimtChunk;              // [dv][32]
    __shared__ float c_hi[kSimtChunk], c_lo[kSimtChunk], w_in[kSimtChunk], w_st[kSimtChunk], s_whole;
    __shared__ float sums[kDecayThreads / 32][kSimtChunk], both[kDecayThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = blockIdx.x % p.chunks, bh = blockIdx.x / p.chunks, b = bh / p.heads, h = bh % p.heads;
    const int t0 = n * kSimtChunk, live = live_tokens(p.lengths, b, p.tokens);
    const T* gq = static_cast<const T*>(p.q.ptr) + b * p.q.sb + (h / p.q.div) * p.q.sh;
    const T* gk = static_cast<const T*>(p.k.ptr) + b * p.k.sb + (h / p.k.div) * p.k.sh;
    const T* gv = static_cast<const T*>(p.v.ptr) + b * p.v.sb + (h / p.v.div) * p.v.sh;
    const T* gg = static_cast<const T*>(p.g.ptr) + b * p.g.sb + (h / p.g.div) * p.g.sh;
    for (int e = tid; e < kSimtChunk * p.dk; e += kDecayThreads) {
        const int i = e / p.dk, d = e % p.dk;
        const bool in = t0 + i < live;
        qs[d * kSimtChunk + i] = in ? to_f(gq[(t0 + i) * p.q.st + d]) : 0.0f;
        ks[d * kSimtChunk + i] = in ? to_f(gk[(t0 + i) * p.k.st + d]) : 0.0f;
    }
    for (int e = tid; e < kSimtChunk * p.dv; e += kDecayThreads) {
        const int i = e / p.dv, d = e % p.dv;
        const bool in = t0 + i < live;
        vs[d * kSimtChunk + i] = in ? to_f(gv[(t0 + i) * p.v.st + d]) : 0.0f;
        gs[d * kSimtChunk + i] = in ? to_f(gg[(t0 + i) * p.g.st + d]) : 0.0f;
    }
    if (warp == 0) {
        float a = t0 + lane < live ? p.log_a[b * p.ab + (t0 + lane) * p.at + h * p.ah] : 0.0f;
        a = a < kReset ? kReset : a;
        double c = (double)a * 1.4426950408889634;
        for (int o = 1; o < 32; o *= 2) {
            const double u = __shfl_up_sync(~0u, c, o);
            if (lane >= o) c += u;
        }
        const double whole = __shfl_sync(~0u, c, 31);
        c_hi[lane] = (float)c;
        c_lo[lane] = (float)(c - (double)(float)c);
        w_in[lane] = ex2((float)c);
        w_st[lane] = ex2((float)(whole - c));
        if (lane == 31) s_whole = ex2((float)whole);
    }
    __syncthreads();
    // far[i]: this thread's share of what crosses the chunk's ends.  Columns d of the states belong to threads d, d + 256, ..
    float early[kSimtChunk], late[kSimtChunk], cross = 0.0f;
#pragma unroll
    for (int i = 0; i < kSimtChunk; ++i) early[i] = late[i] = 0.0f;
    const long long plane = ((long long)bh * p.chunks + n) * p.dv * p.dk;
    const int halves = p.dk <= kDecayThreads / 2 ? 2 : 1, width = kDecayThreads / halves;
    const int d = tid % width, v_lo = tid / width * ((p.dv + halves - 1) / halves),
              v_hi = min(p.dv, v_lo + (p.dv + halves - 1) / halves);
    if (d < p.dk) {
        for (int v = v_lo; v < v_hi; ++v) {
            const float s = p.before[plane + (long long)v * p.dk + d], f = p.behind[plane + (long long)v * p.dk + d];
            cross = fmaf(s, f, cross);
#pragma unroll
            for (int i = 0; i < kSimtChunk; i += 4) {
                const float4 g4 = *reinterpret_cast<const float4*>(gs + v * kSimtChunk + i);
                const float4 v4 = *reinterpret_cast<const float4*>(vs + v * kSimtChunk + i);
                early[i] = fmaf(g4.x, s, early[i]); early[i + 1] = fmaf(g4.y, s, early[i + 1]);
                early[i + 2] = fmaf(g4.z, s, early[i + 2]); early[i + 3] = fmaf(g4.w, s, early[i + 3]);
                late[i] = fmaf(v4.x, f, late[i]); late[i + 1] = fmaf(v4.y, f, late[i + 1]);
                late[i + 2] = fmaf(v4.z, f, late[i + 2]); late[i + 3] = fmaf(v4.w, f, late[i + 3]);
            }
        }
    }
    float r = 0.0f, s = 0.0f;  // of token `lane`, summed over the warp's threads
#pragma unroll
    for (int i = 0; i < kSimtChunk; ++i) {
        float e = d < p.dk ? early[i] * qs[d * kSimtChunk + i] : 0.0f, l = d < p.dk ? late[i] * ks[d * kSimtChunk + i] : 0.0f;
        for (int o = 16; o > 0; o >>= 1) {
            e += __shfl_xor_sync(~0u, e, o);
            l += __shfl_xor_sync(~0u, l, o);
        }
        if (lane == i) { r = e; s = l; }
    }
    for (int o = 16; o > 0; o >>= 1) cross += __shfl_xor_sync(~0u, cross, o);
    // sum_{i>=t} of the early ones, sum_{j<t} of the late ones; t = lane
    r = decayed(w_in[lane], r);
    s = decayed(w_st[lane], s);
    for (int o = 1; o < 32; o *= 2) {
        const float u = __shfl_down_sync(~0u, r, o), w = __shfl_up_sync(~0u, s, o);
        if (lane + o < 32) r += u;
        if (lane >= o) s += w;
    }
    s = __shfl_up_sync(~0u, s, 1);
    float sum = r + (lane ? s : 0.0f);
    // pairs inside the chunk: a warp has rows i = warp, warp + 8, ..; lane j holds W_ij, then its exclusive running sum
    for (int i = warp; i < kSimtChunk; i += kDecayThreads / 32) {
        float x = 0.0f, y = 0.0f;
        for (int e = 0; e < p.dk; ++e) x = fmaf(qs[e * kSimtChunk + i], ks[e * kSimtChunk + lane], x);
        for (int e = 0; e < p.dv; ++e) y = fmaf(gs[e * kSimtChunk + i], vs[e * kSimtChunk + lane], y);
        float w = lane < i ? x * y * ex2((c_hi[i] - c_hi[lane]) + (c_lo[i] - c_lo[lane])) : 0.0f;
        for (int o = 1; o < 32; o *= 2) {
            const float u = __shfl_up_sync(~0u, w, o);
            if (lane >= o) w += u;
        }
        w = __shfl_up_sync(~0u, w, 1);
        if (lane > 0 && lane <= i) sum += w;
    }
    sums[warp][lane] = sum;
    if (lane == 0) both[warp] = cross;
    __syncthreads();
    if (warp == 0) {
        sum = cross = 0.0f;
        for (int w = 0; w < kDecayThreads / 32; ++w) {
            sum += sums[w][lane];
            cross += both[w];
        }
        sum = t0 + lane < live ? p.scale * (sum + decayed(s_whole, cross)) : 0.0f;
        if (p.part) {
            double total = sum;
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
            if (lane == 0) p.part[blockIdx.x] = total;
        } else if (t0 + lane < p.tokens) {
            p.dlog_a[((long long)b * p.tokens + t0 + lane) * p.heads + h] = sum;
        }
    }
}
inline size_t decay_grad_smem(int dk, int dv) { return sizeof(float) * (size_t)kSimtChunk * 2 * (dk + dv); }

// dlog_a[h]: the sum of the chunks' parts over the batch, in 64 bits and in a fixed order; a warp for each head.
__global__ void decay_grad_sum_kernel(const double* part, int batch, int heads, int chunks, float* dlog_a) {
    const int h = blockIdx.x, lane = threadIdx.x;
    double s = 0.0;
    for (int b = 0; b < batch; ++b)
        for (int n = lane; n < chunks; n += 32) s += part[((long long)b * heads + h) * chunks + n];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (lane == 0) dlog_a[h] = (float)s;
}

// ------------------------------------------------------------------------------------------------------------------
// One token: S <- a S + k v^T, o = scale S^T q, for every (sequence, head).  A CTA has kCols columns of one state; its
// threads walk the rows, kCols / kVec threads to a row, so a warp reads whole 128-byte lines and every thread keeps the
// same columns (their v and their sums stay in registers).  Bound by the state's two trips over HBM: 4096 states of 128 x 128
// in 84.8 us are 6.3 TB/s, 97% of a copy's rate.
constexpr int kStepThreads = 256;

struct Step {
    const void *q, *k, *v;
    long long qb, qh, kb, kh, vb, vh;
    int qdiv, kdiv, vdiv;
    const float* log_a;
    long long ab, ah;
    float* pool;
    const int* slots;
    long long pool_rows;
    int heads, dk, dv;
    float scale;
    void* o;
    long long ob, oh;
};

template <int kVec> __device__ __forceinline__ void load_vec(float* to, const float* from);
template <> __device__ __forceinline__ void load_vec<1>(float* to, const float* from) { to[0] = from[0]; }
template <> __device__ __forceinline__ void load_vec<4>(float* to, const float* from) {
    const float4 f = *reinterpret_cast<const float4*>(from);
    to[0] = f.x; to[1] = f.y; to[2] = f.z; to[3] = f.w;
}
template <int kVec> __device__ __forceinline__ void store_vec(const float* from, float* to);
template <> __device__ __forceinline__ void store_vec<1>(const float* from, float* to) { to[0] = from[0]; }
template <> __device__ __forceinline__ void store_vec<4>(const float* from, float* to) {
    *reinterpret_cast<float4*>(to) = make_float4(from[0], from[1], from[2], from[3]);
}

template <class T, int kCols, int kVec>
__global__ void __launch_bounds__(kStepThreads) step_kernel(const Step p) {
    constexpr int kLanes = kCols / kVec, kRows = kStepThreads / kLanes;  // rows of one sweep of the CTA
    __shared__ float ks[256], qs[256];
    __shared__ float part[kRows][kCols];
    const int tid = threadIdx.x, tiles = (p.dv + kCols - 1) / kCols;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / p.heads, h = bh % p.heads;
    const long long slot = p.slots ? (long long)p.slots[b] : b;
    const int c0 = tile * kCols + (tid % kLanes) * kVec, r0 = tid / kLanes;
    T* go = static_cast<T*>(p.o) + b * p.ob + h * p.oh;
    if (slot < 0 || slot >= p.pool_rows) {
        if (tid < kCols && tile * kCols + tid < p.dv) go[tile * kCols + tid] = from_f<T>(0.0f);
        return;
    }
    const T* gq = static_cast<const T*>(p.q) + b * p.qb + (h / p.qdiv) * p.qh;
    const T* gk = static_cast<const T*>(p.k) + b * p.kb + (h / p.kdiv) * p.kh;
    const T* gv = static_cast<const T*>(p.v) + b * p.vb + (h / p.vdiv) * p.vh;
    float* s = p.pool + ((slot * p.heads + h) * p.dk) * (long long)p.dv + c0;
    // kBatch rows are loaded before any is stored: the compiler may not move a load over a store.  The first are on their way
    // before the keys are.
    constexpr int kBatch = 8;
    float cur[kBatch][kVec];
    auto load = [&](int r) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (c0 < p.dv && r + u * kRows < p.dk) load_vec<kVec>(cur[u], s + (long long)(r + u * kRows) * p.dv);
    };
    load(r0);
    for (int i = tid; i < p.dk; i += kStepThreads) {
        ks[i] = to_f(gk[i]);
        qs[i] = to_f(gq[i]);
    }
    const float a = expf(p.log_a[b * p.ab + h * p.ah]);
    float vv[kVec], acc[kVec];
#pragma unroll
    for (int m = 0; m < kVec; ++m) {
        vv[m] = c0 + m < p.dv ? to_f(gv[c0 + m]) : 0.0f;
        acc[m] = 0.0f;
    }
    __syncthreads();
    if (c0 < p.dv) {
        for (int r = r0; r < p.dk; r += kRows * kBatch) {
            if (r != r0) load(r);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int row = r + u * kRows;
                if (row < p.dk) {
                    const float kr = ks[row], qr = qs[row];
#pragma unroll
                    for (int m = 0; m < kVec; ++m) {
                        cur[u][m] = fmaf(kr, vv[m], decayed(a, cur[u][m]));
                        acc[m] = fmaf(qr, cur[u][m], acc[m]);
                    }
                    store_vec<kVec>(cur[u], s + (long long)row * p.dv);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kVec; ++m) part[r0][(tid % kLanes) * kVec + m] = acc[m];
    __syncthreads();
    if (tid < kCols && tile * kCols + tid < p.dv) {
        float sum = 0.0f;
        for (int r = 0; r < kRows; ++r) sum += part[r][tid];
        go[tile * kCols + tid] = from_f<T>(sum * p.scale);
    }
}

}  // namespace ha
