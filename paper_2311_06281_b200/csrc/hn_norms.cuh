// The norms around a block: r = x + scale * gate * norm(branch), y = norm(r), and the gated norm of a block's heads, each
// with its backward pass.  All are bound by HBM: every input element is read once and every output written once, the row
// stays in registers between its reductions, and the gradients that are summed over rows are kept in registers by threads
// that own the same columns of every row they see.
//
// Measured, bf16, and the time of the same bytes at a copy's rate: block, 16384 rows of 2048: forward 69 us (51), backward 154 us
// (82); gated, 16384 x 16 rows of 128: forward 43 us (31), backward 69 us (51); in float32 66 us (61) and 117 us (102).  Between its
// loads and its stores a row waits for two sums over its threads (three on the way back), each some 500 clocks: other rows of the
// SM have to cover that, and how many fit is up to registers.  The backward kernels are short of those: threads with 8 elements of a
// row spill 32 to 84 bytes, rows of 8192 float32 240 bytes (one CTA of 512 threads to an SM: 209 us for 82), the widest rows
// up to 1.4 KB.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace hn {

// at most 16 bytes aligned: float32 weights and sums beside 8 bf16 elements are read as two 16-byte halves
template <class T, int kVec> struct alignas(sizeof(T) * kVec < 16 ? sizeof(T) * kVec : 16) Vec { T v[kVec]; };

// CTAs of a backward kernel that shall be resident on an SM beside one another: 768 threads where a thread has 8 elements of a
// row (84 registers each), so that there are rows in flight while others are at their barriers; 512 where the next row is on
// its way in any case (16384 rows of 2048 bf16: 154 us, 768 threads and their spills 233 us).
__host__ __device__ constexpr int resident(int elems, int row_threads, bool ahead) {
    const int threads = row_threads < 128 ? 128 : row_threads;
    return threads * 2 > 1024 ? 1 : (elems > 8 || ahead ? 512 : 768) / threads;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

struct Norms {
    long long rows, gate_rows;
    int dim;
    bool weights_f32;
    float scale, eps;
    const void *x, *branch, *gate, *pre, *post;
    void *r, *y;                                  // forward
    const void *d_r, *d_y;                        // backward
    void *dx, *dbranch, *dgate;
    float *part_pre, *part_post, *part_gate;      // [units, dim] sums over the rows of a unit
    int splits;                                   // units that share one row of the gate
    long long units;
};

// kRowThreads threads have one row; element (v * kRowThreads + t) * kVec + e is thread t's.
template <class T, int kVec, int kNv, int kRowThreads>
struct Slice {
    static constexpr int kElems = kVec * kNv;
    template <class U>
    static __device__ __forceinline__ void load(float (&to)[kElems], const U* row, int t, int dim) {
#pragma unroll
        for (int v = 0; v < kNv; ++v) {
            const int c = (v * kRowThreads + t) * kVec;
            if (c < dim) {
                const Vec<U, kVec> f = *reinterpret_cast<const Vec<U, kVec>*>(row + c);
#pragma unroll
                for (int e = 0; e < kVec; ++e) to[v * kVec + e] = to_f(f.v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < kVec; ++e) to[v * kVec + e] = 0.0f;
            }
        }
    }
    // weights are of T or float32
    static __device__ __forceinline__ void load_weight(float (&to)[kElems], const void* w, bool f32, int t, int dim) {
        if (f32) load(to, static_cast<const float*>(w), t, dim);
        else load(to, static_cast<const T*>(w), t, dim);
    }
    template <class U>
    static __device__ __forceinline__ void store(const float (&from)[kElems], U* row, int t, int dim) {
#pragma unroll
        for (int v = 0; v < kNv; ++v) {
            const int c = (v * kRowThreads + t) * kVec;
            if (c < dim) {
                Vec<U, kVec> f;
#pragma unroll
                for (int e = 0; e < kVec; ++e) f.v[e] = from_f<U>(from[v * kVec + e]);
                *reinterpret_cast<Vec<U, kVec>*>(row + c) = f;
            }
        }
    }
};

// Do two stages of five tensors, beside the sums of rows that share a CTA, fit what a kernel has without asking for more?
__host__ __device__ constexpr bool ahead_fits(int vec, int nv, int row_threads, int elem) {
    const int threads = row_threads < 128 ? 128 : row_threads;
    return vec * elem == 16 && 2 * 5 * nv * 16 * threads + (row_threads < 128 ? 128 * vec * nv * 4 : 0) <= 47 * 1024;
}

// The rows of a block's backward pass on their way while others are worked on: every thread copies its own 16-byte pieces of the
// next row's tensors to shared memory and reads nobody else's, so no barrier belongs to it.  Two stages, as long as they leave
// room for the CTAs of resident(); wider rows have enough in flight without it (8192 float32: 208 us so, 245 us with one stage).
template <class T, int kVec, int kNv, int kRowThreads>
struct Ahead {
    static constexpr int kThreads = kRowThreads < 128 ? 128 : kRowThreads, kPiece = kNv * 16 * kThreads, kTensors = 5;
    static constexpr bool kOn = ahead_fits(kVec, kNv, kRowThreads, sizeof(T));
    static constexpr int kBytes = kOn ? 2 * kTensors * kPiece : 0;
    static __device__ __forceinline__ void copy(uint8_t* sm, int stage, int tensor, const T* row, int t, int dim) {
#pragma unroll
        for (int v = 0; v < kNv; ++v) {
            const int c = (v * kRowThreads + t) * kVec;
            if (c < dim)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(
                                 sm + (stage * kTensors + tensor) * kPiece + (v * kThreads + threadIdx.x) * 16)),
                             "l"(row + c)
                             : "memory");
        }
    }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void arrived(bool next) {  // this row's, of which the next's may be behind
        if (next) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    static __device__ __forceinline__ void read(float (&to)[kVec * kNv], const uint8_t* sm, int stage, int tensor, int t, int dim) {
#pragma unroll
        for (int v = 0; v < kNv; ++v) {
            const bool in = (v * kRowThreads + t) * kVec < dim;
            Vec<T, kVec> f;
            if (in) f = *reinterpret_cast<const Vec<T, kVec>*>(sm + (stage * kTensors + tensor) * kPiece + (v * kThreads + threadIdx.x) * 16);
#pragma unroll
            for (int e = 0; e < kVec; ++e) to[v * kVec + e] = in ? to_f(f.v[e]) : 0.0f;
        }
    }
};

// Sums over the threads of a row.  Rows of up to 32 threads use shuffles alone; wider ones go through shared memory, one
// barrier each: `turn` picks one of three buffers, so that a thread that is late in one sum is not overtaken two sums on.
template <int kRowThreads, int kN>
__device__ __forceinline__ void row_sum(float (&s)[kN], float* red, int& turn) {
    constexpr int kWidth = kRowThreads < 32 ? kRowThreads : 32;
#pragma unroll
    for (int o = kWidth / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < kN; ++i) s[i] += __shfl_xor_sync(~0u, s[i], o);
    if (kRowThreads > 32) {
        constexpr int kWarps = kRowThreads / 32;
        float* buf = red + turn * 64;
        turn = turn == 2 ? 0 : turn + 1;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < kN; ++i) buf[warp * kN + i] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kN; ++i) s[i] = lane < kWarps ? buf[lane * kN + i] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < kN; ++i) s[i] += __shfl_xor_sync(~0u, s[i], o);
    }
}

// Back through n = x * rs, rs = 1 / sqrt(mean(x^2) + eps): rs * (d - n * mean(d n)).  Over a single element the two terms
// cancel to what eps leaves of them, which is then taken from the formula.
__device__ __forceinline__ float norm_back(float d, float n, float mean, float rs, int dim, float eps) {
    return dim == 1 ? rs * d * (eps * rs * rs) : rs * fmaf(-n, mean, d);
}

// float32 results take the exponential that is good to an ulp over the whole range, of -|z| so that the quotient's divisor lies
// between 1 and 2 (16384 x 16 rows of 128: 70 and 132 us, with the fast one 66 and 130, with a division of any size 72 and 141).
// Beside bf16 the fast one does: its error grows with its argument, to 1e-5 at the largest that is not an infinity, and the result
// is rounded to 2e-3.
template <class T> __device__ __forceinline__ float sigmoid(float z);
template <> __device__ __forceinline__ float sigmoid<float>(float z) {
    const float e = expf(-fabsf(z)), r = __fdividef(1.0f, 1.0f + e);
    return z < 0.0f ? e * r : r;
}
template <> __device__ __forceinline__ float sigmoid<__nv_bfloat16>(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

template <class T, int kVec, int kNv, int kRowThreads>
__global__ void __launch_bounds__(kRowThreads < 128 ? 128 : kRowThreads) block_norms_forward_kernel(const Norms p) {
    using S = Slice<T, kVec, kNv, kRowThreads>;
    constexpr int kE = S::kElems, kRowsPerCta = kRowThreads < 128 ? 128 / kRowThreads : 1;
    __shared__ float red[3 * 64];
    int turn = 0;
    const int t = threadIdx.x % kRowThreads;
    long long row = (long long)blockIdx.x * kRowsPerCta + threadIdx.x / kRowThreads;
    const bool live = row < p.rows;
    if (!live) row = p.rows - 1;  // takes part in the sums of its warp, stores nothing
    const float inv = 1.0f / (float)p.dim;
    float h[kE], x[kE], w[kE];
    S::load(h, static_cast<const T*>(p.branch) + row * p.dim, t, p.dim);
    S::load(x, static_cast<const T*>(p.x) + row * p.dim, t, p.dim);
    if (p.post) {
        float s[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < kE; ++e) s[0] = fmaf(h[e], h[e], s[0]);
        row_sum<kRowThreads>(s, red, turn);
        const float rs = rsqrtf(fmaf(s[0], inv, p.eps));
        S::load_weight(w, p.post, p.weights_f32, t, p.dim);
#pragma unroll
        for (int e = 0; e < kE; ++e) h[e] *= rs * w[e];
    }
    if (p.gate) {
        S::load(w, static_cast<const T*>(p.gate) + (row / p.gate_rows) * p.dim, t, p.dim);
#pragma unroll
        for (int e = 0; e < kE; ++e) h[e] *= w[e];
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        x[e] = fmaf(p.scale, h[e], x[e]);
        s[0] = fmaf(x[e], x[e], s[0]);
    }
    if (live) S::store(x, static_cast<T*>(p.r) + row * p.dim, t, p.dim);
    row_sum<kRowThreads>(s, red, turn);
    const float rs = rsqrtf(fmaf(s[0], inv, p.eps));
    S::load_weight(w, p.pre, p.weights_f32, t, p.dim);
#pragma unroll
    for (int e = 0; e < kE; ++e) x[e] *= rs * w[e];
    if (live) S::store(x, static_cast<T*>(p.y) + row * p.dim, t, p.dim);
}

// The sums over rows are per unit: a unit is a run of rows within one row of the gate (or of all rows, without a broadcast
// gate).  A CTA takes a contiguous run of units and keeps the weights' sums over all of them; only the gate's sum starts
// anew with each unit.
template <class T, int kVec, int kNv, int kRowThreads>
__global__ void __launch_bounds__(kRowThreads < 128 ? 128 : kRowThreads, resident(kVec * kNv, kRowThreads, Ahead<T, kVec, kNv, kRowThreads>::kOn)) block_norms_backward_kernel(const Norms p) {
    using S = Slice<T, kVec, kNv, kRowThreads>;
    constexpr int kE = S::kElems, kRowsPerCta = kRowThreads < 128 ? 128 / kRowThreads : 1;
    using A = Ahead<T, kVec, kNv, kRowThreads>;
    __shared__ float red[3 * 64];
    extern __shared__ __align__(16) uint8_t sm[];
    float* join = reinterpret_cast<float*>(sm + A::kBytes);  // [kRowsPerCta][dim], only where rows share a CTA
    int turn = 0;
    const int t = threadIdx.x % kRowThreads, sub = threadIdx.x / kRowThreads;
    const float inv = 1.0f / (float)p.dim;
    const bool wide_gate = p.gate && p.gate_rows > 1;
    float a_pre[kE] = {}, a_post[kE] = {}, a_gate[kE];

    auto flush = [&](float (&acc)[kE], float* to) {
        if (kRowsPerCta == 1) {
            S::store(acc, to, t, p.dim);
        } else {
            S::store(acc, join + sub * p.dim, t, p.dim);
            __syncthreads();
            for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
                float s = 0.0f;
                for (int i = 0; i < kRowsPerCta; ++i) s += join[i * p.dim + c];
                to[c] = s;
            }
            __syncthreads();
        }
    };
    const long long per_gate = wide_gate ? p.gate_rows : p.rows;
    const long long per_unit = (per_gate + p.splits - 1) / p.splits;
    const long long u0 = p.units * blockIdx.x / gridDim.x, u1 = p.units * (blockIdx.x + 1) / gridDim.x;
    for (long long u = u0; u < u1; ++u) {
        const long long base = u / p.splits * per_gate, first = base + u % p.splits * per_unit;
        const long long last = first + per_unit < base + per_gate ? first + per_unit : base + per_gate;
#pragma unroll
        for (int e = 0; e < kE; ++e) a_gate[e] = 0.0f;
        auto fetch = [&](long long at, int stage) {
            const long long row = at + sub < last ? at + sub : last - 1;
            A::copy(sm, stage, 0, static_cast<const T*>(p.branch) + row * p.dim, t, p.dim);
            A::copy(sm, stage, 1, static_cast<const T*>(p.x) + row * p.dim, t, p.dim);
            A::copy(sm, stage, 2, static_cast<const T*>(p.d_y) + row * p.dim, t, p.dim);
            if (p.gate) A::copy(sm, stage, 3, static_cast<const T*>(p.gate) + (row / p.gate_rows) * p.dim, t, p.dim);
            if (p.d_r) A::copy(sm, stage, 4, static_cast<const T*>(p.d_r) + row * p.dim, t, p.dim);
            A::commit();
        };
        if (A::kOn && first < last) fetch(first, 0);
        int stage = 0;
        for (long long at = first; at < last; at += kRowsPerCta) {
            const bool live = at + sub < last, next = at + kRowsPerCta < last;
            const long long row = live ? at + sub : last - 1;
            float h[kE], x[kE], g[kE], dy[kE], w[kE];
            if constexpr (A::kOn) {
                if (next) fetch(at + kRowsPerCta, stage ^ 1);
                A::arrived(next);
                A::read(h, sm, stage, 0, t, p.dim);
                A::read(x, sm, stage, 1, t, p.dim);
                A::read(dy, sm, stage, 2, t, p.dim);
                if (p.gate) A::read(g, sm, stage, 3, t, p.dim);
                else
#pragma unroll
                    for (int e = 0; e < kE; ++e) g[e] = 1.0f;
            } else {
                S::load(h, static_cast<const T*>(p.branch) + row * p.dim, t, p.dim);
                S::load(x, static_cast<const T*>(p.x) + row * p.dim, t, p.dim);
                S::load(dy, static_cast<const T*>(p.d_y) + row * p.dim, t, p.dim);
                if (p.gate) S::load(g, static_cast<const T*>(p.gate) + (row / p.gate_rows) * p.dim, t, p.dim);
                else
#pragma unroll
                    for (int e = 0; e < kE; ++e) g[e] = 1.0f;
            }
            float rs1 = 1.0f;
            if (p.post) {
                float s[1] = {0.0f};
#pragma unroll
                for (int e = 0; e < kE; ++e) s[0] = fmaf(h[e], h[e], s[0]);
                row_sum<kRowThreads>(s, red, turn);
                rs1 = rsqrtf(fmaf(s[0], inv, p.eps));
                S::load_weight(w, p.post, p.weights_f32, t, p.dim);
#pragma unroll
                for (int e = 0; e < kE; ++e) h[e] *= rs1;  // the norm without its weight from here on
#pragma unroll
                for (int e = 0; e < kE; ++e) x[e] = fmaf(p.scale * g[e], h[e] * w[e], x[e]);
            } else {
#pragma unroll
                for (int e = 0; e < kE; ++e) x[e] = fmaf(p.scale * g[e], h[e], x[e]);
            }
            // x is r now
            S::load_weight(w, p.pre, p.weights_f32, t, p.dim);
            float s2[2] = {0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                s2[0] = fmaf(x[e], x[e], s2[0]);
                s2[1] = fmaf(dy[e] * w[e], x[e], s2[1]);
            }
            row_sum<kRowThreads>(s2, red, turn);
            const float rs2 = rsqrtf(fmaf(s2[0], inv, p.eps)), mean = s2[1] * rs2 * inv;
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                const float m = x[e] * rs2;
                if (live) a_pre[e] = fmaf(dy[e], m, a_pre[e]);
                dy[e] = norm_back(dy[e] * w[e], m, mean, rs2, p.dim, p.eps);
            }
            if (p.d_r) {
                if constexpr (A::kOn) A::read(w, sm, stage, 4, t, p.dim);
                else S::load(w, static_cast<const T*>(p.d_r) + row * p.dim, t, p.dim);
#pragma unroll
                for (int e = 0; e < kE; ++e) dy[e] += w[e];
            }
            // dy is the gradient of r now
            if (live) S::store(dy, static_cast<T*>(p.dx) + row * p.dim, t, p.dim);
#pragma unroll
            for (int e = 0; e < kE; ++e) dy[e] *= p.scale;
            if (p.post) S::load_weight(w, p.post, p.weights_f32, t, p.dim);
            if (p.gate) {
                float dg[kE];
#pragma unroll
                for (int e = 0; e < kE; ++e) dg[e] = dy[e] * h[e] * (p.post ? w[e] : 1.0f);
                if (wide_gate) {
#pragma unroll
                    for (int e = 0; e < kE; ++e) a_gate[e] += live ? dg[e] : 0.0f;
                } else if (live) {
                    S::store(dg, static_cast<T*>(p.dgate) + row * p.dim, t, p.dim);
                }
            }
#pragma unroll
            for (int e = 0; e < kE; ++e) dy[e] *= g[e];
            if (p.post) {
                float s1[1] = {0.0f};
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    if (live) a_post[e] = fmaf(dy[e], h[e], a_post[e]);
                    dy[e] *= w[e];
                    s1[0] = fmaf(dy[e], h[e], s1[0]);
                }
                row_sum<kRowThreads>(s1, red, turn);
#pragma unroll
                for (int e = 0; e < kE; ++e) dy[e] = norm_back(dy[e], h[e], s1[0] * inv, rs1, p.dim, p.eps);
            }
            if (live) S::store(dy, static_cast<T*>(p.dbranch) + row * p.dim, t, p.dim);
            stage ^= 1;
        }
        if (wide_gate) flush(a_gate, p.part_gate + u * p.dim);
    }
    flush(a_pre, p.part_pre + (long long)blockIdx.x * p.dim);
    if (p.post) flush(a_post, p.part_post + (long long)blockIdx.x * p.dim);
}

template <class T, int kVec, int kNv, int kRowThreads>
__global__ void __launch_bounds__(kRowThreads < 128 ? 128 : kRowThreads) gated_norm_forward_kernel(const Norms p) {
    using S = Slice<T, kVec, kNv, kRowThreads>;
    constexpr int kE = S::kElems, kRowsPerCta = kRowThreads < 128 ? 128 / kRowThreads : 1;
    __shared__ float red[3 * 64];
    int turn = 0;
    const int t = threadIdx.x % kRowThreads;
    long long row = (long long)blockIdx.x * kRowsPerCta + threadIdx.x / kRowThreads;
    const bool live = row < p.rows;
    if (!live) row = p.rows - 1;
    float x[kE], g[kE], w[kE];
    S::load(x, static_cast<const T*>(p.x) + row * p.dim, t, p.dim);
    if (p.gate) S::load(g, static_cast<const T*>(p.gate) + row * p.dim, t, p.dim);
    S::load_weight(w, p.pre, p.weights_f32, t, p.dim);
    float s[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < kE; ++e) s[0] = fmaf(x[e], x[e], s[0]);
    row_sum<kRowThreads>(s, red, turn);
    const float rs = rsqrtf(fmaf(s[0], 1.0f / (float)p.dim, p.eps));
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        x[e] *= rs * w[e];
        if (p.gate) x[e] *= g[e] * sigmoid<T>(g[e]);
    }
    if (live) S::store(x, static_cast<T*>(p.y) + row * p.dim, t, p.dim);
}

template <class T, int kVec, int kNv, int kRowThreads>
__global__ void __launch_bounds__(kRowThreads < 128 ? 128 : kRowThreads, resident(kVec * kNv, kRowThreads, false)) gated_norm_backward_kernel(const Norms p) {
    using S = Slice<T, kVec, kNv, kRowThreads>;
    constexpr int kE = S::kElems, kRowsPerCta = kRowThreads < 128 ? 128 / kRowThreads : 1;
    __shared__ float red[3 * 64];
    extern __shared__ float join[];
    int turn = 0;
    const int t = threadIdx.x % kRowThreads, sub = threadIdx.x / kRowThreads;
    const float inv = 1.0f / (float)p.dim;
    float acc[kE] = {}, w[kE];
    S::load_weight(w, p.pre, p.weights_f32, t, p.dim);
    for (long long at = (long long)blockIdx.x * kRowsPerCta; at < p.rows; at += (long long)gridDim.x * kRowsPerCta) {
        const bool live = at + sub < p.rows;
        const long long row = live ? at + sub : p.rows - 1;
        float x[kE], g[kE], dy[kE];
        S::load(x, static_cast<const T*>(p.x) + row * p.dim, t, p.dim);
        S::load(dy, static_cast<const T*>(p.d_y) + row * p.dim, t, p.dim);
        if (p.gate) S::load(g, static_cast<const T*>(p.gate) + row * p.dim, t, p.dim);
        float s[2] = {0.0f, 0.0f};
        float dz[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            float d = dy[e];
            if (p.gate) {
                const float sg = sigmoid<T>(g[e]);
                dz[e] = d * w[e] * sg * fmaf(g[e], 1.0f - sg, 1.0f);  // times the norm below
                d *= g[e] * sg;
            }
            dy[e] = d;  // the gradient of norm * weight
            s[0] = fmaf(x[e], x[e], s[0]);
            s[1] = fmaf(d * w[e], x[e], s[1]);
        }
        row_sum<kRowThreads>(s, red, turn);
        const float rs = rsqrtf(fmaf(s[0], inv, p.eps)), mean = s[1] * rs * inv;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const float n = x[e] * rs;
            if (live) acc[e] = fmaf(dy[e], n, acc[e]);
            dz[e] *= n;
            dy[e] = norm_back(dy[e] * w[e], n, mean, rs, p.dim, p.eps);
        }
        if (live) {
            S::store(dy, static_cast<T*>(p.dx) + row * p.dim, t, p.dim);
            if (p.gate) S::store(dz, static_cast<T*>(p.dgate) + row * p.dim, t, p.dim);
        }
    }
    float* to = p.part_pre + (long long)blockIdx.x * p.dim;
    if (kRowsPerCta == 1) {
        S::store(acc, to, t, p.dim);
    } else {
        S::store(acc, join + sub * p.dim, t, p.dim);
        __syncthreads();
        for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
            float s = 0.0f;
            for (int i = 0; i < kRowsPerCta; ++i) s += join[i * p.dim + c];
            to[c] = s;
        }
    }
}

// out[g, c] = sum over the `per` rows of part that belong to g; a CTA has 32 columns, its warps share the rows in a fixed
// order (32 of them, or 8 where there are few rows).  Two such sums of one shape go in one launch (blockIdx.y).
struct Parts {
    const float* part[2];
    void* out[2];
    long long per;
    int dim;
};
template <class T, int kWarps>
__global__ void __launch_bounds__(32 * kWarps) sum_parts_kernel(const Parts p) {
    __shared__ float s_part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tiles = (p.dim + 31) / 32;
    const int c = blockIdx.x % tiles * 32 + lane;
    const long long g = blockIdx.x / tiles;
    const float* part = p.part[blockIdx.y];
    float s = 0.0f;
    if (c < p.dim) {
#pragma unroll 4
        for (long long i = warp; i < p.per; i += kWarps) s += part[(g * p.per + i) * p.dim + c];
    }
    s_part[warp][lane] = s;
    __syncthreads();
    for (int w = warp; w < 32; w += kWarps) {  // a column each
        s = lane < kWarps ? s_part[lane][w] : 0.0f;
        for (int o = kWarps / 2; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        const int col = blockIdx.x % tiles * 32 + w;
        if (lane == 0 && col < p.dim) static_cast<T*>(p.out[blockIdx.y])[g * p.dim + col] = from_f<T>(s);
    }
}

}  // namespace hn
