// One token of the delta rule for every (sequence, head):  S <- a S,  e = beta (v - S^T k),  S <- S + k e^T,  o = scale S^T q.
// A CTA has kCols columns of one state, all rows of them in registers: the state is read once and written once.  The two sums over
// the rows that depend on the old state, S^T k and S^T q, are formed together, since scale (S + k e^T)^T q = scale (S^T q + (q.k) e):
// one round through shared memory between reading and writing.  Bound by the state's two trips over HBM, and by a CTA's loads, sums
// and stores following each other (four CTAs to an SM): 256 sequences of 16 states of 128 x 128, 94 to 99 us for the 82 of a copy.
// Measured against CTAs of 64 columns and 256 threads (96 us): 128 threads with 32 columns 98, with 64 columns 99, 512 threads with
// 128 columns 107, half the rows to a thread 122 and more (more registers around the state than in it).
#pragma once
#include "ha_common.cuh"

namespace hd {

constexpr int kStepThreads = 256;

struct Step {
    const void *q, *k, *v;
    long long qb, qh, kb, kh, vb, vh;
    int qdiv, kdiv, vdiv;
    const float *log_a, *beta;
    long long ab, ah, bb, bh;
    float* pool;
    const int* slots;
    long long pool_rows;
    int heads, dk, dv;
    float scale;
    void* o;
    long long ob, oh;
};

// kBatch: rows that a thread has, at least ceil(dk / (kStepThreads / (kCols / kVec)))
template <class T, int kCols, int kVec, int kBatch>
__global__ void __launch_bounds__(kStepThreads, kBatch * kVec <= 32 ? 4 : 2) step_kernel(const Step p) {
    constexpr int kLanes = kCols / kVec, kRows = kStepThreads / kLanes;
    __shared__ float ks[256], qs[256], es[kCols];
    __shared__ float part[2][kRows][kCols];
    __shared__ float qk_part[kStepThreads / 32];
    const int tid = threadIdx.x, tiles = (p.dv + kCols - 1) / kCols;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / p.heads, h = bh % p.heads;
    const long long slot = p.slots ? (long long)p.slots[b] : b;
    const int lane = tid % kLanes, c0 = tile * kCols + lane * kVec, r0 = tid / kLanes;
    T* go = static_cast<T*>(p.o) + b * p.ob + h * p.oh;
    if (slot < 0 || slot >= p.pool_rows) {
        if (tid < kCols && tile * kCols + tid < p.dv) go[tile * kCols + tid] = ha::from_f<T>(0.0f);
        return;
    }
    const T* gq = static_cast<const T*>(p.q) + b * p.qb + (h / p.qdiv) * p.qh;
    const T* gk = static_cast<const T*>(p.k) + b * p.kb + (h / p.kdiv) * p.kh;
    const T* gv = static_cast<const T*>(p.v) + b * p.vb + (h / p.vdiv) * p.vh;
    float* s = p.pool + ((slot * p.heads + h) * p.dk) * (long long)p.dv + c0;
    float cur[kBatch][kVec];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const int row = r0 + u * kRows;
        const bool on = row < p.dk && c0 < p.dv;
        if constexpr (kVec == 4) {
            const float4 f = on ? *reinterpret_cast<const float4*>(s + (long long)row * p.dv) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            cur[u][0] = f.x; cur[u][1] = f.y; cur[u][2] = f.z; cur[u][3] = f.w;
        } else {
            cur[u][0] = on ? s[(long long)row * p.dv] : 0.0f;
        }
    }
    const float kt = tid < p.dk ? ha::to_f(gk[tid]) : 0.0f, qt = tid < p.dk ? ha::to_f(gq[tid]) : 0.0f;
    ks[tid] = kt;
    qs[tid] = qt;
    float qk = qt * kt;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) qk += __shfl_xor_sync(~0u, qk, o);
    if (tid % 32 == 0) qk_part[tid / 32] = qk;
    const float a = expf(p.log_a[b * p.ab + h * p.ah]), beta = p.beta[b * p.bb + h * p.bh];
    __syncthreads();
    float sum_k[kVec] = {}, sum_q[kVec] = {};
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const int row = r0 + u * kRows;
        if (row < p.dk) {
            const float kr = ks[row], qr = qs[row];
#pragma unroll
            for (int m = 0; m < kVec; ++m) {
                cur[u][m] = ha::decayed(a, cur[u][m]);
                sum_k[m] = fmaf(kr, cur[u][m], sum_k[m]);
                sum_q[m] = fmaf(qr, cur[u][m], sum_q[m]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kVec; ++m) {
        part[0][r0][lane * kVec + m] = sum_k[m];
        part[1][r0][lane * kVec + m] = sum_q[m];
    }
    __syncthreads();
    if (tid < kCols) {
        const int c = tile * kCols + tid;
        float x = 0.0f, y = 0.0f, z = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            x += part[0][r][tid];
            y += part[1][r][tid];
        }
#pragma unroll
        for (int w = 0; w < kStepThreads / 32; ++w) z += qk_part[w];
        const float e = c < p.dv ? beta * (ha::to_f(gv[c]) - x) : 0.0f;
        es[tid] = e;
        if (c < p.dv) go[c] = ha::from_f<T>(p.scale * fmaf(z, e, y));
    }
    __syncthreads();
    float e[kVec];
#pragma unroll
    for (int m = 0; m < kVec; ++m) e[m] = es[lane * kVec + m];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const int row = r0 + u * kRows;
        if (row < p.dk && c0 < p.dv) {
            const float kr = ks[row];
#pragma unroll
            for (int m = 0; m < kVec; ++m) cur[u][m] = fmaf(kr, e[m], cur[u][m]);
            if constexpr (kVec == 4) *reinterpret_cast<float4*>(s + (long long)row * p.dv) = make_float4(cur[u][0], cur[u][1], cur[u][2], cur[u][3]);
            else s[(long long)row * p.dv] = cur[u][0];
        }
    }
}

}  // namespace hd
