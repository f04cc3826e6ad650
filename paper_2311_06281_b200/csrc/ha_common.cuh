// What the kernels on matrix states share: tensors, the fault record, conversions, bounded waits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ha_ptx.cuh"

namespace ha {

constexpr float kLog2e = 1.4426950408889634f;
// A log decay below this is a reset: e^-10000 is zero in float32 by a wide margin, and clamping -inf to it keeps every
// difference of sums finite.  (x < kReset keeps NaN.)
constexpr float kReset = -1.0e4f;

struct Rows {  // [batch, tokens, heads', dim] with a contiguous last dimension, strides in elements
    const void* ptr;
    long long sb, st, sh;
    int div;  // head h reads head h / div
};

struct Fault {  // the header that heinsen_scan_check() reads
    unsigned long long started_id, error_id;
    int error_code, error_where;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ int live_tokens(const int* lengths, int b, int tokens) {
    if (!lengths) return tokens;
    const int n = lengths[b];
    return n < 0 ? 0 : (n > tokens ? tokens : n);
}

// d * s without 0 * inf: a decay of zero forgets the state whatever it holds
__device__ __forceinline__ float decayed(float d, float s) { return d == 0.0f ? 0.0f : d * s; }

constexpr uint32_t kDrainSpin = 1u << 16;    // polls for what is still in flight when a CTA leaves (0.15 us each, measured)

// A thread whose wait has given up runs on without waiting (its warp's loads and stores of tensor memory need every lane), but
// never arrives on a barrier again: nobody takes what it did not do for done, no barrier gets more arrivals in a phase than it
// expects (one too many makes a fault), and the others' waits find `stop` set.
struct Waiter {
    uint32_t bars;
    volatile int* stop;  // in shared memory: some wait of this CTA gave up
    uint32_t limit;
    __device__ __forceinline__ bool operator()(int bar, int turn) const {
#pragma unroll 1
        for (uint32_t i = 0; i < limit; ++i) {
            if (bar_try(bars + 8 * bar, turn & 1)) return true;
            if (*stop) return false;
        }
        *stop = 1 + bar;
        return false;
    }
    // What this thread has in flight on a barrier lands before it leaves, whoever has given up meanwhile.
    __device__ __forceinline__ void drain(int bar, int turn) const {
#pragma unroll 1
        for (uint32_t i = 0; i < kDrainSpin && !bar_try(bars + 8 * bar, turn & 1); ++i) {}
    }
};

// A pair of values as kTerms bf16 pairs whose sum is the pair.
template <int kTerms>
__device__ __forceinline__ void split(pair v, uint32_t (&t)[kTerms]) {
    t[0] = pack_bf16(v);
#pragma unroll
    for (int i = 1; i < kTerms; ++i) {
        v = minus_bf16(v, t[i - 1]);
        t[i] = pack_bf16(v);
    }
}

}  // namespace ha
