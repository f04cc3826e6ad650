// C ABI of the delta rule with a decay: the gradients.
#include "hd_grad_mma.cuh"
#include "hd_host.h"

namespace {

using namespace hd_host;

// Workspace of a backward call: header | images of the chunks | q, k, v, dO as terms where TMA cannot load them | gradients of each
// head where heads are shared, float32 | states before, their gradients after every chunk | E, F | sums over V | of decay gradients
struct Space {
    size_t image, q, k, v, g, dq, dk, dv, states, gradients, errors, back, dots, part, total;
};
template <int KP, int TI> Space space_of(const heinsen_attention_problem* p) {
    constexpr int C = hd::chunk_tokens(KP), TM = 3;
    const size_t rows = (size_t)p->batch * p->tokens * p->heads, chunks = (size_t)chunks_of(p), slices = (p->v_dim + 15) / 16;
    Space s;
    s.image = kHeaderBytes;
    s.q = s.image + image_bytes<C, TM, TM, true>(p);
    s.k = s.q + terms_bytes(p, view_of(p->q, p->heads, p->q_heads, p->k_dim));
    s.v = s.k + terms_bytes(p, view_of(p->k, p->heads, p->k_heads, p->k_dim));
    s.g = s.v + terms_bytes(p, view_of(p->v, p->heads, p->v_heads, p->v_dim));
    s.dq = s.g + up256((size_t)TI * p->batch * p->tokens * p->heads * ((p->v_dim + 7) / 8 * 8) * 2);  // dO's strides are not known yet
    s.dk = s.dq + (p->q_heads == p->heads ? 0 : up256(rows * p->k_dim * 4));
    s.dv = s.dk + (p->k_heads == p->heads ? 0 : up256(rows * p->k_dim * 4));
    s.states = s.dv + (p->v_heads == p->heads ? 0 : up256(rows * p->v_dim * 4));
    s.gradients = s.states + up256(chunks * slices * 16 * KP * 4);
    s.errors = s.gradients + up256(chunks * slices * 16 * KP * 4);
    s.back = s.errors + up256(chunks * slices * 16 * C * 4);
    s.dots = s.back + up256(chunks * slices * 16 * C * 4);
    s.part = s.dots + up256(chunks * 2 * slices * C * 4);
    s.total = s.part + up256(chunks * 8);
    return s;
}

// To sum the heads that share a gradient's row.
template <class T> void add_sum(hd::Sums* all, const float* from, void* to, const heinsen_attention_problem* p, int groups, int dim) {
    const bool whole = dim % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & (4 * sizeof(T) - 1)) == 0;
    all->tensors[all->count++] = {from, to, p->batch * p->tokens * groups * (whole ? dim / 4 : dim), p->heads / groups, dim, whole};
}
template <class T> hs_status launch_sums(const hd::Sums& all, cudaStream_t stream) {
    if (!all.count) return HS_OK;
    long long most = 0;
    for (int i = 0; i < all.count; ++i) most = std::max(most, all.tensors[i].units);
    const dim3 grid((unsigned)std::min<long long>((most + 255) / 256, kSms * 16), all.count);
    hd::shared_sum_kernel<T><<<grid, 256, 0, stream>>>(all);
    return launched("shared_sum_kernel");
}

template <int KP, int TI, class T>
hs_status launch_back(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mg, const hd::Params& q, int* word, cudaStream_t stream) {
    constexpr int C = hd::chunk_tokens(KP), TM = 3;
    static std::atomic<unsigned long long> done{0};
    return launch_slices<hd::ScanLayout<KP, C, TI, TM, TM, true, true>>(hd::back_kernel<KP, C, TI, TM, T>, done, mq, mk, mg, q, word, stream);
}

// The gradients of the chunks: tcgen05 for bf16 and keys up to 128 wide (4096 chunks, 128 wide: 392 us; with mma.sync 498 us before
// the other was made faster), mma.sync for the rest, where all factors have three terms or the tiles would not fit.
template <int KP, int TI, class T>
hs_status launch_grad(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mg, const hd::Params& q, int* word, cudaStream_t stream) {
    constexpr int C = hd::chunk_tokens(KP), TM = 3;
    static std::atomic<unsigned long long> done{0};
    const unsigned grid = (unsigned)((long long)q.batch * q.heads * q.chunks);
    if constexpr (TI == 1 && KP <= 128) {
        using L = hd::GradMmaLayout<KP>;
        static_assert(L::end <= 232448, "shared memory");
        const auto fn = hd::grad_mma_kernel<KP, T>;
        const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)L::end, done);
        if (st != HS_OK) return st;
        hd::Params g = q;
        CUtensorMap mdq, mdk;
        auto out = [&](CUtensorMap* m, void* to, int each) {  // the tensor map of a gradient that TMA can store
            std::memset(m, 0, sizeof *m);
            const long long sh = q.dk, stk = sh * q.heads;
            const View v{{to, stk * q.tokens, stk, sh, 1}, q.heads, q.dk};
            return !each && tma_strides(v, q.batch, q.tokens) && encode(m, v, q.batch, q.tokens, 64, C);
        };
        g.dq_tma = out(&mdq, q.dq, q.each_q);
        g.dk_tma = out(&mdk, q.dk_out, q.each_k);
        fn<<<std::min(grid, (unsigned)kSms), hd::kGradMmaThreads, L::end, stream>>>(mq, mk, mg, mdq, mdk, g, (int)grid, word);
    } else {
        using L = hd::GradLayout<KP, C, TI, TM>;
        static_assert(L::end <= 232448, "shared memory");
        const auto fn = hd::grad_kernel<KP, C, TI, TM, T>;
        const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)L::end, done);
        if (st != HS_OK) return st;
        fn<<<grid, hd::kGradThreads, L::end, stream>>>(mq, mk, mg, q, word);
    }
    return launched("grad_kernel");
}

template <int KP, class T>
hs_status backward(const heinsen_delta_problem* dp, const heinsen_attention_tensor* d_o, const float* d_state, void* dq, void* dk, void* dv, float* dlog_a,
                   float* dbeta, float* dstate0, uint8_t* ws, cudaStream_t stream) {
    constexpr int C = hd::chunk_tokens(KP), TI = sizeof(T) == 2 ? 1 : 3, TM = 3;
    const heinsen_attention_problem* p = &dp->a;
    const Space sp = space_of<KP, TI>(p);
    int* const word = gave_up_word();
    if (!word) return hs_internal::cuda_fail("cudaGetSymbolAddress", cudaGetLastError());
    if (chunks_of(p) > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    auto at = [&](size_t offset) { return reinterpret_cast<float*>(ws + offset); };
    hd::Params q = params_of(dp, C, ws);
    q.image = ws + sp.image;
    q.states = at(sp.states); q.gradients = at(sp.gradients); q.errors = at(sp.errors); q.errors_back = at(sp.back); q.dots = at(sp.dots);
    CUtensorMap mq, mk, mv, mg;
    hs_status st;
    hd::Terms terms{};
    if ((st = map_of<T, TI>(&mq, p, view_of(p->q, p->heads, p->q_heads, p->k_dim), ws + sp.q, 64, C, &terms)) != HS_OK) return st;
    if ((st = map_of<T, TI>(&mk, p, view_of(p->k, p->heads, p->k_heads, p->k_dim), ws + sp.k, 64, C, &terms)) != HS_OK) return st;
    const bool many = fits_tcgen05<KP, TI>() && many_slices(p, true);
    q.parts = many ? (p->v_dim + 31) / 32 : (p->v_dim + 15) / 16;
    if ((st = map_of<T, TI>(&mv, p, view_of(p->v, p->heads, p->v_heads, p->v_dim), ws + sp.v, many ? 64 : 16, C, &terms)) != HS_OK) return st;
    if ((st = map_of<T, TI>(&mg, p, view_of(*d_o, p->heads, p->heads, p->v_dim), ws + sp.g, 16, C, &terms)) != HS_OK) return st;
    CUtensorMap mg64 = mg;  // the same in tiles of 64 columns
    if (many) {
        View g = view_of(*d_o, p->heads, p->heads, p->v_dim);
        if (terms_bytes(p, g)) {
            const long long sh = (p->v_dim + 7) / 8 * 8, stk = sh * p->heads;
            g = {{ws + sp.g, stk * p->tokens, stk, sh, 1}, p->heads, (int)sh};
        }
        if (!encode(&mg64, g, p->batch, p->tokens, 64, C)) return hs_internal::cuda_fail("cuTensorMapEncodeTiled", cudaErrorInvalidValue);
    }
    if ((st = launch_terms<T, TI>(terms, stream)) != HS_OK) return st;
    if ((st = launch_chunks<KP, C, TI, TM, TM, true>(mq, mk, q, word, stream)) != HS_OK) return st;
    {
        hd::Params f = q;
        f.s_in = p->state0;
        if constexpr (fits_tcgen05<KP, TI>()) st = many ? launch_pass<KP, 1, T>(mq, mk, mv, f, word, stream) : launch_scan<KP, C, TI, TM, TM, false, T>(mq, mk, mv, f, word, stream);
        else st = launch_scan<KP, C, TI, TM, TM, false, T>(mq, mk, mv, f, word, stream);
        if (st != HS_OK) return st;
    }
    {
        hd::Params r = q;
        r.s_in = d_state; r.s_out = dstate0;
        const bool each = p->v_heads != p->heads;
        r.out = each ? ws + sp.dv : dv;
        r.oh = p->v_dim; r.ot = (long long)p->heads * p->v_dim; r.ob = p->tokens * r.ot;
        auto back = [&](auto type) {
            using Out = decltype(type);
            if constexpr (fits_tcgen05<KP, TI>())
                if (many) return launch_pass<KP, 2, Out>(mq, mk, mg64, r, word, stream);
            return launch_back<KP, TI, Out>(mq, mk, mg, r, word, stream);
        };
        st = each ? back(float{}) : back(T{});
        if (st != HS_OK) return st;
        if (each) {
            hd::Sums sums{};
            add_sum<T>(&sums, at(sp.dv), dv, p, p->v_heads, p->v_dim);
            if ((st = launch_sums<T>(sums, stream)) != HS_OK) return st;
        }
    }
    const bool fixed = p->log_a.batch_stride == 0 && p->log_a.token_stride == 0;
    double* const part = reinterpret_cast<double*>(ws + sp.part);
    hd::Params g = q;
    g.dlog_a = fixed ? nullptr : dlog_a;
    g.part = fixed && dlog_a ? part : nullptr;
    g.dbeta = dbeta;
    const bool eq = p->q_heads != p->heads, ek = p->k_heads != p->heads;
    if (eq || ek) {  // both by heads, then: one of the two may be its own sum
        float *wq = at(sp.dq), *wk = at(sp.dk);
        g.dq = eq ? (void*)wq : dq; g.dk_out = ek ? (void*)wk : dk;
        g.each_q = eq; g.each_k = ek;
        if ((st = launch_grad<KP, TI, T>(mq, mk, mg, g, word, stream)) != HS_OK) return st;
        hd::Sums sums{};
        if (eq) add_sum<T>(&sums, wq, dq, p, p->q_heads, p->k_dim);
        if (ek) add_sum<T>(&sums, wk, dk, p, p->k_heads, p->k_dim);
        if ((st = launch_sums<T>(sums, stream)) != HS_OK) return st;
    } else {
        g.dq = dq; g.dk_out = dk;
        if ((st = launch_grad<KP, TI, T>(mq, mk, mg, g, word, stream)) != HS_OK) return st;
    }
    if (g.part) {
        hd::part_sum_kernel<<<(unsigned)p->heads, 32, 0, stream>>>(part, (int)p->batch, p->heads, q.chunks, dlog_a);
        st = launched("part_sum_kernel");
    }
    return st;
}

template <class T>
hs_status backward_of(const heinsen_delta_problem* p, const heinsen_attention_tensor* d_o, const float* d_state, void* dq, void* dk, void* dv, float* dlog_a,
                      float* dbeta, float* dstate0, uint8_t* ws, cudaStream_t s) {
    const int w = width_of(p->a.k_dim);
    return w == 64    ? backward<64, T>(p, d_o, d_state, dq, dk, dv, dlog_a, dbeta, dstate0, ws, s)
           : w == 128 ? backward<128, T>(p, d_o, d_state, dq, dk, dv, dlog_a, dbeta, dstate0, ws, s)
                      : backward<256, T>(p, d_o, d_state, dq, dk, dv, dlog_a, dbeta, dstate0, ws, s);
}

// The gradients of a call without sequences, heads or tokens: zeros wherever they have elements all the same; the state's own is
// that of the last state, through no token.
hs_status no_tokens(const heinsen_delta_problem* dp, const float* d_state, void* dq, void* dk, void* dv, float* dlog_a, float* dstate0, cudaStream_t stream) {
    const heinsen_attention_problem* p = &dp->a;
    const size_t size = p->dtype == HS_F32 ? 4 : 2, rows = (size_t)p->batch * p->tokens, states = (size_t)p->batch * p->heads * p->k_dim * p->v_dim * 4;
    const bool fixed = p->log_a.batch_stride == 0 && p->log_a.token_stride == 0;
    const struct { void* to; size_t bytes; } all[] = {{dq, rows * p->q_heads * p->k_dim * size}, {dk, rows * p->k_heads * p->k_dim * size},
                                                      {dv, rows * p->v_heads * p->v_dim * size}, {dlog_a, fixed ? (size_t)p->heads * 4 : 0},
                                                      {dstate0, d_state ? 0 : states}};
    cudaError_t e = cudaSuccess;
    for (const auto& z : all)
        if (z.to && z.bytes && e == cudaSuccess) e = cudaMemsetAsync(z.to, 0, z.bytes, stream);
    if (e == cudaSuccess && dstate0 && d_state && states) e = cudaMemcpyAsync(dstate0, d_state, states, cudaMemcpyDeviceToDevice, stream);
    return e == cudaSuccess ? HS_OK : hs_internal::cuda_fail("cudaMemsetAsync", e);
}

}  // namespace

namespace hd_host {

size_t backward_bytes(const heinsen_delta_problem* dp) {
    const heinsen_attention_problem* p = &dp->a;
    const int w = width_of(p->k_dim);
    if (p->dtype == HS_F32) return (w == 64 ? space_of<64, 3>(p) : w == 128 ? space_of<128, 3>(p) : space_of<256, 3>(p)).total;
    return (w == 64 ? space_of<64, 1>(p) : w == 128 ? space_of<128, 1>(p) : space_of<256, 1>(p)).total;
}

}  // namespace hd_host

extern "C" hs_status heinsen_delta_backward(const heinsen_delta_problem* p, const heinsen_attention_tensor* d_o, const float* d_state, void* dq, void* dk,
                                            void* dv, float* dlog_a, float* dbeta, float* dstate0, void* workspace, size_t workspace_bytes, void* stream) {
    hs_status st = p ? validate(&p->a) : HS_ERR_INVALID_ARG;
    if (st != HS_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (nothing(&p->a) || p->a.tokens == 0) return no_tokens(p, d_state, dq, dk, dv, dlog_a, dstate0, s);
    if ((st = validate_inputs(&p->a)) != HS_OK) return st;
    if (!p->beta.ptr || !d_o || !d_o->ptr || !dq || !dk || !dv) return HS_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
    if (workspace_bytes < backward_bytes(p)) return HS_ERR_WORKSPACE_TOO_SMALL;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return p->a.dtype == HS_F32 ? backward_of<float>(p, d_o, d_state, dq, dk, dv, dlog_a, dbeta, dstate0, ws, s)
                                : backward_of<__nv_bfloat16>(p, d_o, d_state, dq, dk, dv, dlog_a, dbeta, dstate0, ws, s);
}
