// C ABI of the delta rule with a decay: checks of the arguments, workspace layout, forward pass, one-token step.
#include "hd_host.h"
#include "hd_step.cuh"

__device__ int g_delta_gave_up;

namespace hd_host {

int* gave_up_word() {
    static std::atomic<int*> words[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
    int* w = dev < 64 ? words[dev].load(std::memory_order_relaxed) : nullptr;
    if (w) return w;
    void* at = nullptr;
    if (cudaGetSymbolAddress(&at, g_delta_gave_up) != cudaSuccess) return nullptr;
    if (dev < 64) words[dev].store(static_cast<int*>(at), std::memory_order_relaxed);
    return static_cast<int*>(at);
}

}  // namespace hd_host

namespace {

using namespace hd_host;

// Workspace of a forward call: header | images of the chunks | q, k, v as terms where TMA cannot load them
struct Space {
    size_t image, q, k, v, total;
};
template <int KP, int TI> Space space_of(const heinsen_attention_problem* p) {
    constexpr int C = hd::chunk_tokens(KP), TM = 3, TP = TI == 1 ? 2 : 3;
    Space s;
    s.image = kHeaderBytes;
    s.q = s.image + image_bytes<C, TM, TP, false>(p);
    s.k = s.q + terms_bytes(p, view_of(p->q, p->heads, p->q_heads, p->k_dim));
    s.v = s.k + terms_bytes(p, view_of(p->k, p->heads, p->k_heads, p->k_dim));
    s.total = s.v + terms_bytes(p, view_of(p->v, p->heads, p->v_heads, p->v_dim));
    return s;
}

template <int KP, class T>
hs_status forward(const heinsen_delta_problem* dp, const heinsen_attention_tensor* o, float* state, uint8_t* ws, cudaStream_t stream) {
    constexpr int C = hd::chunk_tokens(KP), TI = sizeof(T) == 2 ? 1 : 3, TM = 3, TP = TI == 1 ? 2 : 3;
    const heinsen_attention_problem* p = &dp->a;
    const Space sp = space_of<KP, TI>(p);
    int* const word = gave_up_word();
    if (!word) return hs_internal::cuda_fail("cudaGetSymbolAddress", cudaGetLastError());
    if (chunks_of(p) > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    hd::Params q = params_of(dp, C, ws);
    q.image = ws + sp.image;
    q.s_in = p->state0; q.s_out = state;
    q.out = const_cast<void*>(o->ptr); q.ob = o->batch_stride; q.ot = o->token_stride; q.oh = o->head_stride;
    const bool many = fits_tcgen05<KP, TI>() && many_slices(p, false);
    CUtensorMap mq, mk, mv;
    hs_status st;
    hd::Terms terms{};
    if (p->tokens) {
        if ((st = map_of<T, TI>(&mq, p, view_of(p->q, p->heads, p->q_heads, p->k_dim), ws + sp.q, 64, C, &terms)) != HS_OK) return st;
        if ((st = map_of<T, TI>(&mk, p, view_of(p->k, p->heads, p->k_heads, p->k_dim), ws + sp.k, 64, C, &terms)) != HS_OK) return st;
        if ((st = map_of<T, TI>(&mv, p, view_of(p->v, p->heads, p->v_heads, p->v_dim), ws + sp.v, many ? 64 : 16, C, &terms)) != HS_OK) return st;
        if ((st = launch_terms<T, TI>(terms, stream)) != HS_OK) return st;
        if ((st = launch_chunks<KP, C, TI, TM, TP, false>(mq, mk, q, word, stream)) != HS_OK) return st;
    } else {
        std::memset(&mq, 0, sizeof mq);
        mk = mv = mq;  // no chunk is loaded
    }
    if constexpr (fits_tcgen05<KP, TI>())
        if (many) return launch_pass<KP, 0, T>(mq, mk, mv, q, word, stream);
    return launch_scan<KP, C, TI, TM, TP, true, T>(mq, mk, mv, q, word, stream);
}

template <class T>
hs_status forward_of(const heinsen_delta_problem* dp, const heinsen_attention_tensor* o, float* state, uint8_t* ws, cudaStream_t stream) {
    const int w = width_of(dp->a.k_dim);
    return w == 64 ? forward<64, T>(dp, o, state, ws, stream) : w == 128 ? forward<128, T>(dp, o, state, ws, stream)
                                                              : forward<256, T>(dp, o, state, ws, stream);
}

size_t forward_bytes(const heinsen_attention_problem* p) {
    const int w = width_of(p->k_dim);
    if (p->dtype == HS_F32) return (w == 64 ? space_of<64, 3>(p) : w == 128 ? space_of<128, 3>(p) : space_of<256, 3>(p)).total;
    return (w == 64 ? space_of<64, 1>(p) : w == 128 ? space_of<128, 1>(p) : space_of<256, 1>(p)).total;
}

template <class T>
hs_status step(const hd::Step& s, long long batch, cudaStream_t stream) {
    const bool vec = s.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(s.pool) & 15u) == 0;
    auto go = [&](auto fn, int cols) {
        const long long grid = batch * s.heads * ((s.dv + cols - 1) / cols);
        if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
        fn<<<(unsigned)grid, hd::kStepThreads, 0, stream>>>(s);
        return launched("step_kernel");
    };
    if (!vec) return go(hd::step_kernel<T, 32, 1, 32>, 32);
    // 32 columns to a CTA where 64 would be two CTAs for each SM or fewer: states of 128 x 128, 32 CTAs of 64 columns 6.2 us, their columns in
    // 32s 4.1; 128 CTAs 6.2, 5.1; 256 CTAs 6.2, 6.2; 512 CTAs 8.4, 8.3; 1024 CTAs 12.6, 14.4.
    const bool narrow = s.dv <= 32 || batch * s.heads * ((s.dv + 63) / 64) <= 2 * kSms;
    if (narrow) return s.dk <= 128 ? go(hd::step_kernel<T, 32, 4, 4>, 32) : go(hd::step_kernel<T, 32, 4, 8>, 32);
    return s.dk <= 128 ? go(hd::step_kernel<T, 64, 4, 8>, 64) : go(hd::step_kernel<T, 64, 4, 16>, 64);
}

}  // namespace

extern "C" {

size_t heinsen_delta_workspace_bytes(const heinsen_delta_problem* p, int backward) {
    if (!p || validate(&p->a) != HS_OK) return 0;
    if (nothing(&p->a)) return kHeaderBytes;
    return backward ? backward_bytes(p) : forward_bytes(&p->a);
}

hs_status heinsen_delta_forward(const heinsen_delta_problem* p, const heinsen_attention_tensor* o, float* state, void* workspace,
                                size_t workspace_bytes, void* stream) {
    hs_status st = p ? validate(&p->a) : HS_ERR_INVALID_ARG;
    if (st != HS_OK || nothing(&p->a)) return st;
    if ((st = validate_inputs(&p->a)) != HS_OK) return st;
    if (!o || (p->a.tokens && (!o->ptr || !p->beta.ptr))) return HS_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
    if (workspace_bytes < forward_bytes(&p->a)) return HS_ERR_WORKSPACE_TOO_SMALL;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return p->a.dtype == HS_F32 ? forward_of<float>(p, o, state, ws, s) : forward_of<__nv_bfloat16>(p, o, state, ws, s);
}

hs_status heinsen_delta_check(void* stream) {
    int sms, where = 0;
    const hs_status st = hs_internal::current_device(&sms);
    if (st != HS_OK) return st;
    cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaStreamSynchronize", e);
    e = cudaMemcpyFromSymbol(&where, g_delta_gave_up, sizeof where);
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaMemcpyFromSymbol", e);
    if (!where) return HS_OK;
    const int none = 0;
    e = cudaMemcpyToSymbol(g_delta_gave_up, &none, sizeof none);
    return e == cudaSuccess ? HS_ERR_COPY_TIMEOUT : hs_internal::cuda_fail("cudaMemcpyToSymbol", e);
}

hs_status heinsen_delta_step(const heinsen_delta_problem* dp, const heinsen_attention_tensor* o, float* pool_state, int64_t pool,
                             const int32_t* slots, void* stream) {
    hs_status st = dp ? validate(&dp->a) : HS_ERR_INVALID_ARG;
    if (st != HS_OK) return st;
    const heinsen_attention_problem* p = &dp->a;
    if (p->tokens != 1 || p->lengths || p->state0 || pool < 0) return HS_ERR_INVALID_ARG;
    if (!slots && pool < p->batch) return HS_ERR_INVALID_ARG;
    if (nothing(p)) return HS_OK;
    if ((st = validate_inputs(p)) != HS_OK) return st;
    if (!dp->beta.ptr || !o || !o->ptr || (pool && !pool_state)) return HS_ERR_INVALID_ARG;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    hd::Step s;
    s.q = p->q.ptr; s.k = p->k.ptr; s.v = p->v.ptr;
    s.qb = p->q.batch_stride; s.qh = p->q.head_stride; s.qdiv = p->heads / p->q_heads;
    s.kb = p->k.batch_stride; s.kh = p->k.head_stride; s.kdiv = p->heads / p->k_heads;
    s.vb = p->v.batch_stride; s.vh = p->v.head_stride; s.vdiv = p->heads / p->v_heads;
    s.log_a = static_cast<const float*>(p->log_a.ptr); s.ab = p->log_a.batch_stride; s.ah = p->log_a.head_stride;
    s.beta = static_cast<const float*>(dp->beta.ptr); s.bb = dp->beta.batch_stride; s.bh = dp->beta.head_stride;
    s.pool = pool_state; s.slots = slots; s.pool_rows = pool;
    s.heads = p->heads; s.dk = p->k_dim; s.dv = p->v_dim; s.scale = p->scale;
    s.o = const_cast<void*>(o->ptr); s.ob = o->batch_stride; s.oh = o->head_stride;
    cudaStream_t str = static_cast<cudaStream_t>(stream);
    return p->dtype == HS_F32 ? step<float>(s, p->batch, str) : step<__nv_bfloat16>(s, p->batch, str);
}

}  // extern "C"
