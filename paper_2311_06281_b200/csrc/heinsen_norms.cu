// C ABI of the norms around a block: checks of the arguments, choice of the row layout, launches.
#include "../../include/heinsen_attention.h"

#include <algorithm>
#include <cmath>
#include <cstring>

#include "hn_norms.cuh"
#include "hs_internal.h"

namespace {

using hn::Norms;
constexpr long long kMaxRows = 1ll << 40;
constexpr int kMaxDim = 16384;
enum Which { kBlockForward, kBlockBackward, kGatedForward, kGatedBackward };

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// Does every row of every tensor start on 16 bytes?
bool vectors_fit(const heinsen_norms_problem* p, std::initializer_list<const void*> ptrs) {
    if ((p->dim * (p->dtype == HS_F32 ? 4 : 2)) % 16) return false;
    uintptr_t bits = 0;
    for (const void* q : ptrs) bits |= reinterpret_cast<uintptr_t>(q);
    // a weight in float32 is read 8 elements (32 bytes) at a time beside bf16 rows; two 16-byte loads, 16-byte aligned
    return (bits & 15) == 0;
}

// Rows are laid over threads so that one thread has 4 to 16 elements (float32) or 8 to 16 (bf16): fewer leave the sums
// over a row's threads dominant, more do not fit the registers of the backward pass, which keeps three running sums and
// four rows of its slice.  Measured at 2048 bf16: 256 threads to a row 69 us forward and 168 us backward (without the copies
// ahead), a warp to a row 102 us and 230 us.
struct Layout { int vec, nv, threads; };
Layout choose(int dim, bool f32, bool vectors) {
    if (!vectors) {
        if (dim <= 128) return {1, 4, 32};
        if (dim <= 512) return {1, 4, 128};
        if (dim <= 2048) return {1, 4, 512};
        if (dim <= 4096) return {1, 4, 1024};
        return {1, 16, 1024};
    }
    const int vec = f32 ? 4 : 8, n = dim / vec;
    if (n <= 8) return {vec, 1, 8};
    if (n <= 16) return {vec, 1, 16};
    if (n <= 32) return {vec, 1, 32};
    if (n <= 64) return {vec, 2, 32};
    if (n <= 128) return {vec, 1, 128};
    if (n <= 256) return {vec, 1, 256};
    if (n <= 512) return {vec, 2, 256};
    if (n <= 1024) return {vec, 2, 512};
    if (n <= 2048) return {vec, 4, 512};
    return {vec, 4, 1024};
}

struct Kernel { const void* fn; size_t smem; };  // beside the rows that share a CTA
template <class T, int kVec, int kNv, int kThreads>
Kernel pick(Which w) {
    switch (w) {
        case kBlockForward: return {(const void*)hn::block_norms_forward_kernel<T, kVec, kNv, kThreads>, 0};
        case kBlockBackward:
            return {(const void*)hn::block_norms_backward_kernel<T, kVec, kNv, kThreads>, hn::Ahead<T, kVec, kNv, kThreads>::kBytes};
        case kGatedForward: return {(const void*)hn::gated_norm_forward_kernel<T, kVec, kNv, kThreads>, 0};
        case kGatedBackward: return {(const void*)hn::gated_norm_backward_kernel<T, kVec, kNv, kThreads>, 0};
    }
    return {nullptr, 0};
}
template <class T, int kVec>
Kernel kernel_for(Which w, const Layout& l) {
    if (l.vec == 1) {
        if (l.threads == 32) return pick<T, 1, 4, 32>(w);
        if (l.threads == 128) return pick<T, 1, 4, 128>(w);
        if (l.threads == 512) return pick<T, 1, 4, 512>(w);
        return l.nv == 4 ? pick<T, 1, 4, 1024>(w) : pick<T, 1, 16, 1024>(w);
    }
    switch (l.threads) {
        case 8: return pick<T, kVec, 1, 8>(w);
        case 16: return pick<T, kVec, 1, 16>(w);
        case 32: return l.nv == 1 ? pick<T, kVec, 1, 32>(w) : pick<T, kVec, 2, 32>(w);
        case 128: return pick<T, kVec, 1, 128>(w);
        case 256: return l.nv == 1 ? pick<T, kVec, 1, 256>(w) : pick<T, kVec, 2, 256>(w);
        case 512: return l.nv == 2 ? pick<T, kVec, 2, 512>(w) : pick<T, kVec, 4, 512>(w);
    }
    if constexpr (kVec == 4) return pick<T, kVec, 4, 1024>(w);
    return {nullptr, 0};  // 8 elements a vector: 512 threads of 4 already hold the widest row
}
Kernel kernel_for(Which w, const Layout& l, bool f32) {
    return f32 ? kernel_for<float, 4>(w, l) : kernel_for<__nv_bfloat16, 8>(w, l);
}

hs_status launch(const Kernel& k, const Norms& n, long long grid, int threads, size_t smem, cudaStream_t stream) {
    Norms copy = n;
    void* args[] = {&copy};
    const cudaError_t e = cudaLaunchKernel(k.fn, dim3((unsigned)grid), dim3((unsigned)threads), args, smem + k.smem, stream);
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaLaunchKernel (norms)", e);
    hs_internal::count_launches(1);
    return HS_OK;
}

// What does not depend on the pointers, but for whether there is a gate.
hs_status validate_sizes(const heinsen_norms_problem* p, bool block) {
    if (!p || p->rows < 0 || p->rows > kMaxRows || p->dim < 1 || p->dim > kMaxDim) return HS_ERR_INVALID_ARG;
    if ((p->dtype != HS_F32 && p->dtype != HS_BF16) || (p->weight_dtype != HS_F32 && p->weight_dtype != p->dtype))
        return HS_ERR_INVALID_ARG;
    if (!std::isfinite(p->eps) || p->eps < 0.0f || (block && !std::isfinite(p->scale))) return HS_ERR_INVALID_ARG;
    if (p->rows > (1ll << 46) / p->dim) return HS_ERR_INVALID_ARG;
    if (block && p->gate && (p->gate_rows < 1 || p->rows % p->gate_rows)) return HS_ERR_INVALID_ARG;
    return HS_OK;
}
hs_status validate(const heinsen_norms_problem* p, bool block) {
    const hs_status st = validate_sizes(p, block);
    if (st != HS_OK || p->rows == 0) return st;
    if (!p->x || !p->pre_weight || (block && !p->branch)) return HS_ERR_INVALID_ARG;
    return HS_OK;
}

Norms make(const heinsen_norms_problem* p) {
    Norms n;
    std::memset(&n, 0, sizeof n);
    n.rows = p->rows;
    n.gate_rows = p->gate ? std::max<int64_t>(1, p->gate_rows) : 1;
    n.dim = p->dim;
    n.weights_f32 = p->weight_dtype == HS_F32;
    n.scale = p->scale;
    n.eps = p->eps;
    n.x = p->x; n.branch = p->branch; n.gate = p->gate; n.pre = p->pre_weight; n.post = p->post_weight;
    return n;
}

// CTAs of the backward kernels, which stay and sum over their rows: as many as are resident at once.  Every CTA leaves one row
// of partial sums behind.
long long stay(long long rows, const Layout& l, bool ahead) {
    const int threads = std::max(128, l.threads), per_cta = threads / l.threads;
    const long long most = 148ll * std::max(1, hn::resident(l.vec * l.nv, l.threads, ahead));
    return std::max(1ll, std::min(most, (rows + per_cta - 1) / per_cta));
}

// How the rows of a block's backward pass are cut into units (see the kernel).
void cut(const heinsen_norms_problem* p, const Layout& l, long long* units, int* splits, long long* grid) {
    const long long want = stay(p->rows, l, hn::ahead_fits(l.vec, l.nv, l.threads, p->dtype == HS_F32 ? 4 : 2));
    const bool wide = p->gate && p->gate_rows > 1;
    const long long gates = wide ? p->rows / p->gate_rows : 1, per_gate = wide ? p->gate_rows : p->rows;
    // whole rows of the gate to each CTA where there are enough of them, else each is split
    long long s = gates >= want ? 1 : std::min(per_gate, want / gates);
    const long long per_unit = (per_gate + s - 1) / s;
    s = (per_gate + per_unit - 1) / per_unit;  // no empty units
    *splits = (int)s;
    *units = gates * s;
    *grid = std::min(*units, want);
}

size_t block_parts(const heinsen_norms_problem* p, const Layout& l, size_t* gate_at) {
    long long units, grid;
    int splits;
    cut(p, l, &units, &splits, &grid);
    const size_t weights = 2 * up256((size_t)grid * p->dim * 4);
    *gate_at = weights;
    return weights + (p->gate && p->gate_rows > 1 ? up256((size_t)units * p->dim * 4) : 0);
}

// One or two (out2 not NULL) sums of the same shape.
hs_status sum_parts(const float* part, void* out, const float* part2, void* out2, long long groups, long long per, int dim, bool f32,
                    cudaStream_t stream) {
    const long long grid = groups * ((dim + 31) / 32);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    const hn::Parts parts{{part, part2}, {out, out2}, per, dim};
    const dim3 g((unsigned)grid, out2 ? 2 : 1);
    const bool few = per <= 64;
    if (f32 && few) hn::sum_parts_kernel<float, 8><<<g, 256, 0, stream>>>(parts);
    else if (f32) hn::sum_parts_kernel<float, 32><<<g, 1024, 0, stream>>>(parts);
    else if (few) hn::sum_parts_kernel<__nv_bfloat16, 8><<<g, 256, 0, stream>>>(parts);
    else hn::sum_parts_kernel<__nv_bfloat16, 32><<<g, 1024, 0, stream>>>(parts);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaLaunchKernel (sum of parts)", e);
    hs_internal::count_launches(1);
    return HS_OK;
}

hs_status forward(Which which, const heinsen_norms_problem* p, void* r, void* y, void* stream) {
    const bool block = which == kBlockForward;
    hs_status st = validate(p, block);
    if (st != HS_OK || p->rows == 0) return st;
    if (!y || (block && !r)) return HS_ERR_INVALID_ARG;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    Norms n = make(p);
    n.r = r; n.y = y;
    const bool f32 = p->dtype == HS_F32;
    const Layout l = choose(p->dim, f32, vectors_fit(p, {p->x, block ? p->branch : nullptr, p->gate, p->pre_weight,
                                                         block ? p->post_weight : nullptr, r, y}));
    const int threads = std::max(128, l.threads);
    const long long grid = (p->rows + threads / l.threads - 1) / (threads / l.threads);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    return launch(kernel_for(which, l, f32), n, grid, threads, 0, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

hs_status heinsen_block_norms_forward(const heinsen_norms_problem* p, void* r, void* y, void* stream) {
    return forward(kBlockForward, p, r, y, stream);
}
hs_status heinsen_gated_norm_forward(const heinsen_norms_problem* p, void* y, void* stream) {
    return forward(kGatedForward, p, nullptr, y, stream);
}

size_t heinsen_block_norms_workspace_bytes(const heinsen_norms_problem* p) {
    if (validate_sizes(p, true) != HS_OK) return 0;
    if (p->rows == 0) return 256;
    // the larger of the two layouts the pointers may lead to
    size_t at;
    const bool f32 = p->dtype == HS_F32;
    return std::max(block_parts(p, choose(p->dim, f32, false), &at),
                    p->dim * (f32 ? 4 : 2) % 16 ? 0 : block_parts(p, choose(p->dim, f32, true), &at));
}

hs_status heinsen_block_norms_backward(const heinsen_norms_problem* p, const void* d_r, const void* d_y, void* dx,
                                       void* dbranch, void* dgate, void* dpre, void* dpost, void* workspace,
                                       size_t workspace_bytes, void* stream_) {
    hs_status st = validate(p, true);
    if (st != HS_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool f32 = p->dtype == HS_F32, w32 = p->weight_dtype == HS_F32;
    if (!dpre || (p->post_weight && !dpost)) return HS_ERR_INVALID_ARG;
    int sms;
    if (p->rows > 0) {
        if (!d_y || !dx || !dbranch || (p->gate && !dgate)) return HS_ERR_INVALID_ARG;
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
        if (workspace_bytes < heinsen_block_norms_workspace_bytes(p)) return HS_ERR_WORKSPACE_TOO_SMALL;
    }
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    if (p->rows == 0) {
        cudaError_t e = cudaMemsetAsync(dpre, 0, (size_t)p->dim * (w32 ? 4 : 2), stream);
        if (e == cudaSuccess && p->post_weight) e = cudaMemsetAsync(dpost, 0, (size_t)p->dim * (w32 ? 4 : 2), stream);
        return e == cudaSuccess ? HS_OK : hs_internal::cuda_fail("cudaMemsetAsync", e);
    }
    const bool wide = p->gate && p->gate_rows > 1;
    const Layout l = choose(p->dim, f32, vectors_fit(p, {p->x, p->branch, p->gate, p->pre_weight, p->post_weight, d_r, d_y, dx,
                                                         dbranch, wide ? nullptr : dgate}));
    Norms n = make(p);
    n.d_r = d_r; n.d_y = d_y; n.dx = dx; n.dbranch = dbranch; n.dgate = dgate;
    long long grid;
    cut(p, l, &n.units, &n.splits, &grid);
    size_t gate_at;
    block_parts(p, l, &gate_at);
    n.part_pre = static_cast<float*>(workspace);
    n.part_post = n.part_pre + up256((size_t)grid * p->dim * 4) / 4;
    n.part_gate = n.part_pre + gate_at / 4;
    const int threads = std::max(128, l.threads), sub = threads / l.threads;
    st = launch(kernel_for(kBlockBackward, l, f32), n, grid, threads, sub > 1 ? (size_t)sub * p->dim * 4 : 0, stream);
    if (st == HS_OK)
        st = sum_parts(n.part_pre, dpre, n.part_post, p->post_weight ? dpost : nullptr, 1, grid, p->dim, w32, stream);
    if (st == HS_OK && wide)
        st = sum_parts(n.part_gate, dgate, nullptr, nullptr, p->rows / p->gate_rows, n.splits, p->dim, f32, stream);
    return st;
}

size_t heinsen_gated_norm_workspace_bytes(const heinsen_norms_problem* p) {
    if (validate_sizes(p, false) != HS_OK) return 0;
    const bool f32 = p->dtype == HS_F32;
    const long long grid = std::max(stay(p->rows, choose(p->dim, f32, false), false),
                                    p->dim * (f32 ? 4 : 2) % 16 ? 1 : stay(p->rows, choose(p->dim, f32, true), false));
    return up256((size_t)grid * p->dim * 4);
}

hs_status heinsen_gated_norm_backward(const heinsen_norms_problem* p, const void* d_y, void* dx, void* dgate, void* dweight,
                                      void* workspace, size_t workspace_bytes, void* stream_) {
    hs_status st = validate(p, false);
    if (st != HS_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool f32 = p->dtype == HS_F32, w32 = p->weight_dtype == HS_F32;
    if (!dweight) return HS_ERR_INVALID_ARG;
    if (p->rows > 0) {
        if (!d_y || !dx || (p->gate && !dgate)) return HS_ERR_INVALID_ARG;
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
        if (workspace_bytes < heinsen_gated_norm_workspace_bytes(p)) return HS_ERR_WORKSPACE_TOO_SMALL;
    }
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    if (p->rows == 0) {
        const cudaError_t e = cudaMemsetAsync(dweight, 0, (size_t)p->dim * (w32 ? 4 : 2), stream);
        return e == cudaSuccess ? HS_OK : hs_internal::cuda_fail("cudaMemsetAsync", e);
    }
    const Layout l = choose(p->dim, f32, vectors_fit(p, {p->x, p->gate, p->pre_weight, d_y, dx, dgate}));
    Norms n = make(p);
    n.d_y = d_y; n.dx = dx; n.dgate = dgate;
    n.part_pre = static_cast<float*>(workspace);
    const long long grid = stay(p->rows, l, false);
    const int threads = std::max(128, l.threads), sub = threads / l.threads;
    st = launch(kernel_for(kGatedBackward, l, f32), n, grid, threads, sub > 1 ? (size_t)sub * p->dim * 4 : 0, stream);
    if (st == HS_OK) st = sum_parts(n.part_pre, dweight, nullptr, nullptr, 1, grid, p->dim, w32, stream);
    return st;
}

}  // extern "C"
