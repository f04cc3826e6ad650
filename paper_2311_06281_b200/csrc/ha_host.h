// What the entry points on matrix states share on the host: checks of a problem's sizes, launches, tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "../../include/heinsen_attention.h"
#include "ha_common.cuh"
#include "hs_internal.h"

namespace ha_host {

using ha::Rows;

constexpr long long kMaxTokens = (1ll << 31) - (1ll << 20);
constexpr int kMaxHeadDim = 256;
constexpr size_t kHeaderBytes = 256;

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

inline hs_status validate(const heinsen_attention_problem* p) {
    if (!p || p->batch < 0 || p->tokens < 0 || p->tokens > kMaxTokens) return HS_ERR_INVALID_ARG;
    if (p->heads < 0 || p->q_heads < 0 || p->k_heads < 0 || p->v_heads < 0) return HS_ERR_INVALID_ARG;
    if (p->k_dim < 1 || p->k_dim > kMaxHeadDim || p->v_dim < 1 || p->v_dim > kMaxHeadDim) return HS_ERR_INVALID_ARG;
    if (p->dtype != HS_F32 && p->dtype != HS_BF16) return HS_ERR_INVALID_ARG;
    if (!std::isfinite(p->scale) || p->scale == 0.0f) return HS_ERR_INVALID_ARG;
    if (p->heads > 0) {
        if (!p->q_heads || !p->k_heads || !p->v_heads) return HS_ERR_INVALID_ARG;
        if (p->heads % p->q_heads || p->heads % p->k_heads || p->heads % p->v_heads) return HS_ERR_INVALID_ARG;
        if (p->batch > 0x7fffffffll / p->heads) return HS_ERR_INVALID_ARG;
        if (p->tokens && p->batch > (1ll << 62) / p->tokens / p->heads / std::max(p->k_dim, p->v_dim)) return HS_ERR_INVALID_ARG;
    }
    return HS_OK;
}
inline bool nothing(const heinsen_attention_problem* p) { return p->batch == 0 || p->heads == 0; }
inline hs_status validate_inputs(const heinsen_attention_problem* p) {
    if (p->tokens && (!p->q.ptr || !p->k.ptr || !p->v.ptr || !p->log_a.ptr)) return HS_ERR_INVALID_ARG;
    return HS_OK;
}

inline Rows rows_of(const heinsen_attention_tensor& t, int heads, int own) {
    return {t.ptr, t.batch_stride, t.token_stride, t.head_stride, heads / own};
}

inline hs_status launched(const char* what) {
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return hs_internal::cuda_fail(what, e);
    hs_internal::count_launches(1);
    return HS_OK;
}

// Asks once for each kernel and device: a call costs more host time than a launch.  `done`: bits of the devices, the kernel's own.
// `smem` is the most that any launch of the kernel takes: the limit is the kernel's, and a smaller one set for this call would
// refuse the launch of another thread's.
inline hs_status allow_smem(const void* fn, int smem, std::atomic<unsigned long long>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaGetDevice", e);
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return HS_OK;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaFuncSetAttribute", e);
    done.fetch_or(bit, std::memory_order_relaxed);
    return HS_OK;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeFn encode_fn() {
    static EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}

}  // namespace ha_host
