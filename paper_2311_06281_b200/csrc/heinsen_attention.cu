// C ABI of the attention with a decay for each head: checks of the arguments, workspace layout, launches.
#include "../../include/heinsen_attention.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "ha_host.h"
#include "ha_mma.cuh"
#include "ha_simt.cuh"

namespace {

using namespace ha_host;
using ha::Pass;
using ha::Rows;

constexpr int kSms = 148;  // B200; sizes workspaces the same wherever they are asked for

// Columns of the state that a CTA has, and the CTAs for a state.  64 take fewer reads of shared memory for a product than 32
// (two rows share each), and half of them would idle where a state has no more than 32.
int simt_cols(int dz) { return dz > 32 ? 64 : 32; }
int simt_tiles(int dz) { return (dz + simt_cols(dz) - 1) / simt_cols(dz); }

// Segments of a sequence on the CUDA cores, as below: up to two CTAs for an SM, where cutting in two steps (states, then the
// rest) is less than walking all chunks.  Measured, whole and cut: 24 states of 64 x 64, 31 chunks 230 us and 71 us, 4 chunks
// 37 us and 28 us; 64 of them, 32 chunks 231 us and 152 us; 128 of them 233 us and 257 us (not cut).
int simt_segments(const heinsen_attention_problem* p, int passes) {
    const long long ctas = passes * p->batch * p->heads * simt_tiles(std::max(p->k_dim, p->v_dim));
    const long long chunks = (p->tokens + ha::kSimtChunk - 1) / ha::kSimtChunk;
    const long long most = std::max(1ll, std::min(2 * kSms / std::max(1ll, ctas), chunks));
    const long long each = std::max(1ll, (chunks + most - 1) / most);
    return 2 * each + 1 < chunks ? (int)((chunks + each - 1) / each) : 1;
}
size_t simt_segment_bytes(const heinsen_attention_problem* p, int passes) {
    const long long pairs = p->batch * p->heads;
    const int n = simt_segments(p, passes);
    return n > 1 ? passes * (up256((size_t)pairs * n * p->k_dim * p->v_dim * 4) + up256((size_t)pairs * n * 4)) : 0;
}

template <class T, class OutT, bool kStateOnly>
hs_status simt_launch(const ha::Passes& ps, int n, cudaStream_t stream) {
    int dx = 0, dz = 0;
    for (int i = 0; i < n; ++i) {
        dx = std::max(dx, ps.p[i].dx);
        dz = std::max(dz, ps.p[i].dz);
    }
    const int cols = simt_cols(dz), segments = ps.p[0].segments;
    const size_t smem = ha::simt_pass_smem(dx, cols);
    const auto fn = cols == 64 ? ha::simt_pass_kernel<T, OutT, kStateOnly, 64> : ha::simt_pass_kernel<T, OutT, kStateOnly, 32>;
    static std::atomic<unsigned long long> done[2] = {};
    const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)ha::simt_pass_smem(kMaxHeadDim, cols), done[cols == 64]);
    if (st != HS_OK) return st;
    const long long grid = (long long)ps.p[0].batch * ps.p[0].heads * simt_tiles(dz) * (kStateOnly ? segments - 1 : segments);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    fn<<<dim3((unsigned)grid, (unsigned)n), ha::kSimtThreads, smem, stream>>>(ps);
    return launched("simt_pass_kernel");
}

// n passes over the same sequences, with their segments; `space`: n times simt_segment_bytes() of scratch.
template <class T, class OutT>
hs_status simt_passes(ha::Passes ps, int n, int segments, uint8_t* space, cudaStream_t stream) {
    const long long pairs = (long long)ps.p[0].batch * ps.p[0].heads, plane = (long long)ps.p[0].dx * ps.p[0].dz;
    const int chunks = (ps.p[0].tokens + ha::kSimtChunk - 1) / ha::kSimtChunk;
    const size_t states = up256((size_t)pairs * segments * plane * 4), decays = up256((size_t)pairs * segments * 4);
    for (int i = 0; i < n; ++i) {
        Pass& p = ps.p[i];
        p.segments = segments;
        p.seg_chunks = (chunks + segments - 1) / segments;
        p.seg_state = reinterpret_cast<float*>(space + i * (states + decays));
        p.seg_decay = reinterpret_cast<float*>(space + i * (states + decays) + states);
    }
    if (segments > 1) {
        hs_status st = simt_launch<T, float, true>(ps, n, stream);
        if (st != HS_OK) return st;
        ha::join_passes_kernel<<<dim3((unsigned)(pairs * ((plane + 255) / 256)), (unsigned)n), 256, 0, stream>>>(ps);
        if ((st = launched("join_passes_kernel")) != HS_OK) return st;
    }
    return simt_launch<T, OutT, false>(ps, n, stream);
}

Pass common(const heinsen_attention_problem* p) {
    Pass ps;
    std::memset(&ps, 0, sizeof ps);
    ps.log_a = static_cast<const float*>(p->log_a.ptr);
    ps.ab = p->log_a.batch_stride; ps.at = p->log_a.token_stride; ps.ah = p->log_a.head_stride;
    ps.lengths = p->lengths;
    ps.batch = (int)p->batch; ps.tokens = (int)p->tokens; ps.heads = p->heads;
    ps.scale = p->scale;
    ps.s_in_mul = ps.s_out_mul = 1.0f;
    return ps;
}

// ---- the tensor-core passes
struct View {  // one [batch, tokens, heads', dim] tensor of a pass
    Rows rows;
    int own_heads, dim;
};

// Can TMA address it?  16-byte base and strides; a stride of a dimension of one is never used.
bool tma_fits(const View& v, long long batch, long long tokens) {
    const long long s[3] = {v.own_heads > 1 ? v.rows.sh : 8, tokens > 1 ? v.rows.st : 8, batch > 1 ? v.rows.sb : 8};
    for (long long x : s)
        if (x <= 0 || x % 8 || x >= (1ll << 38)) return false;
    return v.dim % 8 == 0 && v.dim <= 128 && (reinterpret_cast<uintptr_t>(v.rows.ptr) & 15u) == 0;
}
bool encode(CUtensorMap* m, const View& v, long long batch, long long tokens) {
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)v.dim, (cuuint64_t)v.own_heads, (cuuint64_t)tokens, (cuuint64_t)batch};
    const cuuint64_t any = 256;
    const cuuint64_t strides[3] = {v.own_heads > 1 ? (cuuint64_t)v.rows.sh * 2 : any, tokens > 1 ? (cuuint64_t)v.rows.st * 2 : any,
                                   batch > 1 ? (cuuint64_t)v.rows.sb * 2 : any};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)ha::kChunk, 1}, one[4] = {1, 1, 1, 1};
    for (int again = 0;; ++again) {
        const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(v.rows.ptr), dims, strides, box, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r == CUDA_SUCCESS || again) return r == CUDA_SUCCESS;
        cudaFree(nullptr);  // a thread that has made no runtime call yet has no context for the driver's
    }
}

// Segments of a sequence.  Fewer (batch, head) pairs than SMs leave the rest of the GPU idle, so a sequence is cut into as many
// segments as there are SMs for; their states are formed first, from keys and values alone, and joined.  Measured at dimension
// 128 (and 64), whole against cut: 12 us + 3.9 us a chunk (9 + 3.2) against 35 us + 7 us for each chunk of a segment (29 + 5.5),
// so a cut pays from chunks > 2 each + 5 at either width.  On both sides of that: 64 pairs of 64 chunks 261 us whole, 257 us in two
// (213, 208; not cut); 49 pairs of 16 chunks 75 us, in three 79 us (61, 64; not cut) and of 32 133 us, 116 us (111, 93); 37 pairs
// of 12 chunks 58 us, in four 59 us (48, 48); 16 pairs of 8 chunks 42 us, in eight 40 us (35, 36); 8 pairs of 6 chunks 34 us, in
// six 38 us (29, 34; not cut) and of 8 42 us, 38 us (35, 32); 8 pairs of 64 chunks 246 us, in sixteen 63 us (211, 50).
int segments_for(long long pairs, long long tokens, int sms) {
    const long long chunks = (tokens + ha::kChunk - 1) / ha::kChunk;
    const long long most = std::max(1ll, std::min(sms / std::max(1ll, pairs), chunks));
    const long long each = std::max(1ll, (chunks + most - 1) / most);
    return 2 * each + 5 < chunks ? (int)((chunks + each - 1) / each) : 1;
}
size_t segment_bytes(const heinsen_attention_problem* p) {
    const long long pairs = p->batch * p->heads;
    const int n = segments_for(pairs, p->tokens, kSms);
    return n > 1 ? up256((size_t)pairs * n * p->k_dim * p->v_dim * 4) + up256((size_t)pairs * n * 4) : 0;
}

template <bool kRev, bool kDots, class Out, bool kStateOnly>
hs_status mma_launch(const CUtensorMap& mx, const CUtensorMap& my, const CUtensorMap& mz, const CUtensorMap& mo,
                     const CUtensorMap& mw, const ha::MmaPass& mp, long long pairs, cudaStream_t stream) {
    const auto fn = ha::mma_pass_kernel<kRev, kDots, Out, kStateOnly>;
    const int smem = (int)ha::MmaLayout<kDots>::end;
    static std::atomic<unsigned long long> done{0};
    const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), smem, done);
    if (st != HS_OK) return st;
    const long long grid = pairs * (kStateOnly ? mp.segments - 1 : mp.segments);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    fn<<<(unsigned)grid, ha::kMmaThreads, smem, stream>>>(mx, my, mz, mo, mw, mp);
    return launched("mma_pass_kernel");
}

// What the passes leave for the decay gradients.
struct Dots {
    View w;
    double* near;
    float* far;
    float4* dump;
    float* cross;
};

// One pass, with its segments.  `ws`: workspace header, `space`: segment_bytes() of scratch.
template <bool kRev, bool kDots, class Out>
hs_status mma_pass(const Pass& ps, const View& x, const View& y, const View& z, uint8_t* ws, uint8_t* space, unsigned long long id,
                   cudaStream_t stream, const Dots* dots = nullptr) {
    CUtensorMap mx, my, mz, mo, mw;
    const View o{{ps.out, ps.ob, ps.ot, ps.oh, 1}, ps.heads, ps.dz};
    if (sizeof(Out) == 2 && !encode(&mo, o, ps.batch, ps.tokens))
        return hs_internal::cuda_fail("cuTensorMapEncodeTiled", cudaErrorInvalidValue);
    if (sizeof(Out) != 2) std::memset(&mo, 0, sizeof mo);  // not read
    if (!dots) std::memset(&mw, 0, sizeof mw);
    else if (!encode(&mw, dots->w, ps.batch, ps.tokens)) return hs_internal::cuda_fail("cuTensorMapEncodeTiled", cudaErrorInvalidValue);
    if (!encode(&mx, x, ps.batch, ps.tokens) || !encode(&my, y, ps.batch, ps.tokens) || !encode(&mz, z, ps.batch, ps.tokens))
        return hs_internal::cuda_fail("cuTensorMapEncodeTiled", cudaErrorInvalidValue);
    ha::MmaPass mp;
    std::memset(&mp, 0, sizeof mp);
    mp.log_a = ps.log_a; mp.ab = ps.ab; mp.at = ps.at; mp.ah = ps.ah; mp.lengths = ps.lengths;
    mp.tokens = ps.tokens; mp.heads = ps.heads; mp.dx = ps.dx; mp.dz = ps.dz;
    mp.xdiv = ps.x.div; mp.ydiv = ps.y.div; mp.zdiv = ps.z.div;
    mp.scale = ps.scale;
    mp.s_in = ps.s_in; mp.s_out = ps.s_out; mp.s_in_t = ps.s_in_t;
    mp.s_in_mul = ps.s_in_mul; mp.s_out_mul = ps.s_out_mul;
    mp.out = ps.out; mp.ob = ps.ob; mp.ot = ps.ot; mp.oh = ps.oh;
    mp.fault = reinterpret_cast<ha::Fault*>(ws); mp.call_id = id;
    mp.spin = hs_internal::spin_limit();
    mp.mute = (int)std::min<long long>(hs_internal::mute_tile(), 0x7fffffff);
    const long long pairs = (long long)ps.batch * ps.heads, chunks = (ps.tokens + ha::kChunk - 1) / ha::kChunk;
    mp.segments = segments_for(pairs, ps.tokens, kSms);
    mp.seg_chunks = (int)((chunks + mp.segments - 1) / mp.segments);
    mp.chunks = (int)chunks;
    if (dots) {
        mp.wdiv = dots->w.rows.div; mp.dots = dots->near; mp.dots_far = dots->far; mp.dump = dots->dump; mp.cross = dots->cross;
    }
    if (mp.segments > 1) {
        mp.seg_state = reinterpret_cast<float*>(space);
        mp.seg_decay = reinterpret_cast<float*>(space + up256((size_t)pairs * mp.segments * ps.dx * ps.dz * 4));
        hs_status st = mma_launch<kRev, false, __nv_bfloat16, true>(mx, my, mz, mo, mw, mp, pairs, stream);
        if (st != HS_OK) return st;
        ha::join_segments_kernel<<<(unsigned)(pairs * ((ps.dx * ps.dz + 255) / 256)), 256, 0, stream>>>(mp);
        if ((st = launched("join_segments_kernel")) != HS_OK) return st;
    }
    return mma_launch<kRev, kDots, Out, false>(mx, my, mz, mo, mw, mp, pairs, stream);
}

// The rule for the tensor cores: bf16, head dimensions that TMA can load (multiples of 8, at most 128, 16-byte strides).
bool mma_fits(const heinsen_attention_problem* p) {
    if (p->dtype != HS_BF16 || p->tokens == 0) return false;
    return tma_fits({rows_of(p->q, p->heads, p->q_heads), p->q_heads, p->k_dim}, p->batch, p->tokens) &&
           tma_fits({rows_of(p->k, p->heads, p->k_heads), p->k_heads, p->k_dim}, p->batch, p->tokens) &&
           tma_fits({rows_of(p->v, p->heads, p->v_heads), p->v_heads, p->v_dim}, p->batch, p->tokens);
}
View view_of(const heinsen_attention_tensor& t, int heads, int own, int dim) { return {rows_of(t, heads, own), own, dim}; }

// Workspace of a backward call on the tensor cores: header | segments of a pass | a contiguous dO where TMA cannot load the
// given one | gradients of each head where heads are shared, float32 | dots of the tokens | states before the chunks | their
// products with the gradients behind them | sums of the decay gradients.
struct MmaSpace {
    size_t segments, d_o, dq, dk, dv, dots, dump, cross, part, total;
};
MmaSpace mma_space(const heinsen_attention_problem* p) {
    MmaSpace s;
    const size_t rows = (size_t)p->batch * p->tokens * p->heads, pairs = (size_t)p->batch * p->heads;
    const size_t chunks = pairs * ((p->tokens + ha::kChunk - 1) / ha::kChunk);
    s.segments = kHeaderBytes;
    s.d_o = s.segments + segment_bytes(p);
    s.dq = s.d_o + up256(rows * p->v_dim * 2);
    s.dk = s.dq + (p->q_heads == p->heads ? 0 : up256(rows * p->k_dim * 4));
    s.dv = s.dk + (p->k_heads == p->heads ? 0 : up256(rows * p->k_dim * 4));
    s.dots = s.dv + (p->v_heads == p->heads ? 0 : up256(rows * p->v_dim * 4));
    s.dump = s.dots + up256(4 * rows * 8 + 4 * rows * 4);
    s.cross = s.dump + chunks * 65536;
    s.part = s.cross + up256(chunks * 32);
    s.total = s.part + up256(chunks * 8);
    return s;
}

// Workspace of a backward pass: header | segments of a pass | dq, dk, dv for each head, float32 | the states before every chunk and the gradients
// of the states behind it | sums of the decay gradients.
struct BackwardSpace {
    size_t segments, dq, dk, dv, before, behind, part, total;
};
BackwardSpace backward_space(const heinsen_attention_problem* p) {
    BackwardSpace s;
    const size_t rows = (size_t)p->batch * p->tokens * p->heads;
    const size_t chunks = (size_t)p->batch * p->heads * ((p->tokens + ha::kSimtChunk - 1) / ha::kSimtChunk);
    s.segments = kHeaderBytes;
    s.dq = s.segments + simt_segment_bytes(p, 3);
    s.dk = s.dq + up256(rows * p->k_dim * 4);
    s.dv = s.dk + up256(rows * p->k_dim * 4);
    s.before = s.dv + up256(rows * p->v_dim * 4);
    s.behind = s.before + up256(chunks * p->k_dim * p->v_dim * 4);
    s.part = s.behind + up256(chunks * p->k_dim * p->v_dim * 4);
    s.total = s.part + up256(chunks * 8);
    return s;
}

template <class T>
hs_status forward_pass(const heinsen_attention_problem* p, const heinsen_attention_tensor* o, float* state, uint8_t* ws,
                       cudaStream_t stream) {
    Pass ps = common(p);
    ps.x = rows_of(p->q, p->heads, p->q_heads);
    ps.y = rows_of(p->k, p->heads, p->k_heads);
    ps.z = rows_of(p->v, p->heads, p->v_heads);
    ps.dx = p->k_dim; ps.dz = p->v_dim;
    ps.s_in = p->state0; ps.s_out = state;
    ps.out = const_cast<void*>(o->ptr); ps.ob = o->batch_stride; ps.ot = o->token_stride; ps.oh = o->head_stride;
    if (mma_fits(p) && tma_fits(view_of(*o, p->heads, p->heads, p->v_dim), p->batch, p->tokens))
        return mma_pass<false, false, __nv_bfloat16>(ps, {ps.x, p->q_heads, p->k_dim}, {ps.y, p->k_heads, p->k_dim},
                                                 {ps.z, p->v_heads, p->v_dim}, ws, ws + kHeaderBytes, hs_internal::call_id(), stream);
    ha::Passes list;
    std::memset(&list, 0, sizeof list);
    list.p[0] = ps;
    list.p[0].fault = reinterpret_cast<ha::Fault*>(ws);
    list.p[0].call_id = hs_internal::call_id();
    return simt_passes<T, T>(list, 1, simt_segments(p, 1), ws + kHeaderBytes, stream);
}

template <class T>
hs_status sum_heads(const float* src, void* dst, const heinsen_attention_problem* p, int groups, int dim, cudaStream_t stream) {
    const long long total = (long long)p->batch * p->tokens * groups * dim;
    if (total == 0) return HS_OK;
    const long long grid = std::min<long long>((total + 255) / 256, 148 * 16);
    ha::sum_heads_kernel<T><<<(unsigned)grid, 256, 0, stream>>>(src, static_cast<T*>(dst), p->lengths, (int)p->tokens, p->heads,
                                                               groups, dim, total);
    return launched("sum_heads_kernel");
}

template <class T>
hs_status backward_passes(const heinsen_attention_problem* p, const heinsen_attention_tensor* d_o, const float* d_state,
                          void* dq, void* dk, void* dv, float* dlog_a, float* dstate0, uint8_t* ws,
                          cudaStream_t stream) {
    const BackwardSpace sp = backward_space(p);
    float *wq = reinterpret_cast<float*>(ws + sp.dq), *wk = reinterpret_cast<float*>(ws + sp.dk),
          *wv = reinterpret_cast<float*>(ws + sp.dv);
    float *before = dlog_a ? reinterpret_cast<float*>(ws + sp.before) : nullptr,
          *behind = dlog_a ? reinterpret_cast<float*>(ws + sp.behind) : nullptr;
    double* part = reinterpret_cast<double*>(ws + sp.part);
    ha::Passes list;  // dq, dk, dv
    uint8_t* space = ws + sp.segments;
    const Rows q = rows_of(p->q, p->heads, p->q_heads), k = rows_of(p->k, p->heads, p->k_heads),
               v = rows_of(p->v, p->heads, p->v_heads), g = rows_of(*d_o, p->heads, p->heads);
    hs_status st;
    auto to = [&](Pass& ps, float* w, int dim) {
        ps.out = w; ps.oh = dim; ps.ot = (long long)p->heads * dim; ps.ob = p->tokens * ps.ot;
    };
    {
        Pass ps = common(p);
        ps.x = g; ps.y = v; ps.z = k; ps.dx = p->v_dim; ps.dz = p->k_dim;
        ps.s_in = p->state0; ps.s_in_t = 1;
        to(ps, wq, p->k_dim);
        ps.dump = before;
        list.p[0] = ps;
    }
    {
        Pass ps = common(p);
        ps.x = v; ps.y = g; ps.z = q; ps.dx = p->v_dim; ps.dz = p->k_dim;
        ps.s_in = d_state; ps.s_in_t = 1; ps.s_in_mul = 1.0f / p->scale;  // the scale comes back with the output
        to(ps, wk, p->k_dim);
        ps.dump = behind;
        ps.rev = 1;
        list.p[1] = ps;
    }
    {
        Pass ps = common(p);
        ps.x = k; ps.y = q; ps.z = g; ps.dx = p->k_dim; ps.dz = p->v_dim;
        ps.s_in = d_state; ps.s_in_mul = 1.0f / p->scale;
        ps.s_out = dstate0; ps.s_out_mul = p->scale;
        to(ps, wv, p->v_dim);
        ps.rev = 1;
        list.p[2] = ps;
    }
    list.p[0].fault = reinterpret_cast<ha::Fault*>(ws);
    list.p[0].call_id = hs_internal::call_id();
    if ((st = simt_passes<T, float>(list, 3, simt_segments(p, 3), space, stream)) != HS_OK) return st;
    if ((st = sum_heads<T>(wq, dq, p, p->q_heads, p->k_dim, stream)) != HS_OK) return st;
    if ((st = sum_heads<T>(wk, dk, p, p->k_heads, p->k_dim, stream)) != HS_OK) return st;
    if ((st = sum_heads<T>(wv, dv, p, p->v_heads, p->v_dim, stream)) != HS_OK) return st;
    if (dlog_a) {
        ha::DecayGrad d;
        d.q = q; d.k = k; d.v = v; d.g = g;
        d.log_a = static_cast<const float*>(p->log_a.ptr);
        d.ab = p->log_a.batch_stride; d.at = p->log_a.token_stride; d.ah = p->log_a.head_stride;
        d.lengths = p->lengths; d.tokens = (int)p->tokens; d.heads = p->heads; d.dk = p->k_dim; d.dv = p->v_dim;
        d.chunks = (int)((p->tokens + ha::kSimtChunk - 1) / ha::kSimtChunk);
        d.scale = p->scale; d.before = before; d.behind = behind;
        const bool fixed = p->log_a.batch_stride == 0 && p->log_a.token_stride == 0;
        d.dlog_a = dlog_a; d.part = fixed ? part : nullptr;
        const long long grid = p->batch * p->heads * d.chunks;
        if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
        if (grid) {
            const size_t smem = ha::decay_grad_smem(p->k_dim, p->v_dim);
            static std::atomic<unsigned long long> done{0};
            st = allow_smem(reinterpret_cast<const void*>(ha::decay_grad_kernel<T>), (int)ha::decay_grad_smem(kMaxHeadDim, kMaxHeadDim), done);
            if (st != HS_OK) return st;
            ha::decay_grad_kernel<T><<<(unsigned)grid, ha::kDecayThreads, smem, stream>>>(d);
            if ((st = launched("decay_grad_kernel")) != HS_OK) return st;
        }
        if (fixed) {
            ha::decay_grad_sum_kernel<<<(unsigned)p->heads, 32, 0, stream>>>(part, (int)p->batch, p->heads, d.chunks, dlog_a);
            if ((st = launched("decay_grad_sum_kernel")) != HS_OK) return st;
        }
    }
    return HS_OK;
}

// One gradient: straight into `to` where no head is shared, else a float32 row for each head first.
template <bool kRev, bool kDots>
hs_status gradient(Pass ps, const View& x, const View& y, const View& z, const heinsen_attention_problem* p, int groups, void* to,
                   float* each, uint8_t* ws, unsigned long long id, cudaStream_t stream, const Dots* dots = nullptr) {
    ps.x = x.rows; ps.y = y.rows; ps.z = z.rows; ps.dx = x.dim; ps.dz = z.dim;
    ps.oh = z.dim; ps.ot = (long long)p->heads * z.dim; ps.ob = p->tokens * ps.ot;
    uint8_t* space = ws + kHeaderBytes;
    if (groups == p->heads) {
        ps.out = to;
        return mma_pass<kRev, kDots, __nv_bfloat16>(ps, x, y, z, ws, space, id, stream, dots);
    }
    ps.out = each;
    const hs_status st = mma_pass<kRev, kDots, float>(ps, x, y, z, ws, space, id, stream, dots);
    return st != HS_OK ? st : sum_heads<__nv_bfloat16>(each, to, p, groups, z.dim, stream);
}

template <bool kDots>
hs_status mma_backward(const heinsen_attention_problem* p, const heinsen_attention_tensor* d_o, const float* d_state, void* dq,
                       void* dk, void* dv, float* dlog_a, float* dstate0, uint8_t* ws, cudaStream_t stream) {
    const MmaSpace sp = mma_space(p);
    const unsigned long long id = hs_internal::call_id();
    const int chunks = (int)((p->tokens + ha::kChunk - 1) / ha::kChunk);
    const long long rows = (long long)p->batch * p->tokens * p->heads, pairs = (long long)p->batch * p->heads;
    if (pairs * chunks > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    hs_status st;
    View g = view_of(*d_o, p->heads, p->heads, p->v_dim);
    if (!tma_fits(g, p->batch, p->tokens)) {
        __nv_bfloat16* packed = reinterpret_cast<__nv_bfloat16*>(ws + sp.d_o);
        const long long total = rows * p->v_dim;
        ha::pack_rows_kernel<<<(unsigned)std::min<long long>((total + 255) / 256, kSms * 16), 256, 0, stream>>>(
            g.rows, packed, (int)p->tokens, p->heads, p->v_dim, total);
        if ((st = launched("pack_rows_kernel")) != HS_OK) return st;
        const long long sh = p->v_dim, stk = sh * p->heads;
        g.rows = {packed, stk * p->tokens, stk, sh, 1};
    }
    const View q = view_of(p->q, p->heads, p->q_heads, p->k_dim), k = view_of(p->k, p->heads, p->k_heads, p->k_dim),
               v = view_of(p->v, p->heads, p->v_heads, p->v_dim);
    double* near = reinterpret_cast<double*>(ws + sp.dots);  // [pass][half][token]
    float* far = reinterpret_cast<float*>(near + 4 * rows);
    float4* dump = reinterpret_cast<float4*>(ws + sp.dump);
    float* cross = reinterpret_cast<float*>(ws + sp.cross);
    auto each = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
    {
        Pass ps = common(p);
        ps.s_in = p->state0; ps.s_in_t = 1;
        const Dots d{q, near, far, dump, nullptr};
        if ((st = gradient<false, kDots>(ps, g, v, k, p, p->q_heads, dq, each(sp.dq), ws, id, stream, kDots ? &d : nullptr)) != HS_OK)
            return st;
    }
    {
        Pass ps = common(p);
        ps.s_in = d_state; ps.s_in_t = 1; ps.s_in_mul = 1.0f / p->scale;  // the scale comes back with the output
        const Dots d{k, near + 2 * rows, far + 2 * rows, dump, cross};
        if ((st = gradient<true, kDots>(ps, v, g, q, p, p->k_heads, dk, each(sp.dk), ws, id, stream, kDots ? &d : nullptr)) != HS_OK)
            return st;
    }
    {
        Pass ps = common(p);
        ps.s_in = d_state; ps.s_in_mul = 1.0f / p->scale;
        ps.s_out = dstate0; ps.s_out_mul = p->scale;
        if ((st = gradient<true, false>(ps, k, q, g, p, p->v_heads, dv, each(sp.dv), ws, id, stream)) != HS_OK) return st;
    }
    if (!dlog_a) return HS_OK;
    const bool fixed = p->log_a.batch_stride == 0 && p->log_a.token_stride == 0;
    double* part = reinterpret_cast<double*>(ws + sp.part);
    ha::join_decay_grad_kernel<<<(unsigned)(pairs * chunks), ha::kChunk, 0, stream>>>(
        near, near + 2 * rows, far, far + 2 * rows, cross, static_cast<const float*>(p->log_a.ptr), p->log_a.batch_stride,
        p->log_a.token_stride, p->log_a.head_stride, p->lengths, (int)p->tokens, p->heads, chunks, rows, p->scale,
        fixed ? nullptr : dlog_a, fixed ? part : nullptr);
    if ((st = launched("join_decay_grad_kernel")) != HS_OK || !fixed) return st;
    ha::decay_grad_sum_kernel<<<(unsigned)p->heads, 32, 0, stream>>>(part, (int)p->batch, p->heads, chunks, dlog_a);
    return launched("decay_grad_sum_kernel");
}

// The gradients of a call without sequences or without heads: zeros, wherever they have elements all the same.
hs_status zero_gradients(const heinsen_attention_problem* p, void* dq, void* dk, void* dv, float* dlog_a, cudaStream_t stream) {
    const size_t size = p->dtype == HS_F32 ? 4 : 2, rows = (size_t)p->batch * p->tokens;
    const bool fixed = p->log_a.batch_stride == 0 && p->log_a.token_stride == 0;
    const struct { void* to; size_t bytes; } all[] = {{dq, rows * p->q_heads * p->k_dim * size}, {dk, rows * p->k_heads * p->k_dim * size},
                                                      {dv, rows * p->v_heads * p->v_dim * size},
                                                      {dlog_a, fixed ? (size_t)p->heads * 4 : 0}};
    for (const auto& z : all) {
        if (!z.to || !z.bytes) continue;
        const cudaError_t e = cudaMemsetAsync(z.to, 0, z.bytes, stream);
        if (e != cudaSuccess) return hs_internal::cuda_fail("cudaMemsetAsync", e);
    }
    return HS_OK;
}

hs_status check_space(const heinsen_attention_problem* p, int backward, void* workspace, size_t bytes) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
    return bytes < heinsen_attention_workspace_bytes(p, backward) ? HS_ERR_WORKSPACE_TOO_SMALL : HS_OK;
}

template <class T>
hs_status step(const ha::Step& s, long long batch, cudaStream_t stream) {
    const bool vec = s.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(s.pool) & 15u) == 0;
    auto go = [&](auto fn, int cols) {
        const long long grid = batch * s.heads * ((s.dv + cols - 1) / cols);
        if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
        fn<<<(unsigned)grid, ha::kStepThreads, 0, stream>>>(s);
        return launched("step_kernel");
    };
    if (!vec) return go(ha::step_kernel<T, 32, 1>, 32);
    // 64 columns: two 128-byte lines of a row and eight loads in flight for each of 4 CTAs of an SM (4096 states of 128 x 128:
    // 84.8 us, 32 columns 113.5 us, 128 columns 86.0 us).  32 where there are no more, or where CTAs would be too few for half
    // of the SMs (16 states of 128 x 128: 7.4 us, 64 columns 8.2 us).
    const bool narrow = s.dv <= 32 || batch * s.heads * ((s.dv + 63) / 64) <= kSms / 2;
    return narrow ? go(ha::step_kernel<T, 32, 4>, 32) : go(ha::step_kernel<T, 64, 4>, 64);
}

}  // namespace

extern "C" {

size_t heinsen_attention_workspace_bytes(const heinsen_attention_problem* p, int backward) {
    if (validate(p) != HS_OK) return 0;
    if (nothing(p)) return kHeaderBytes;
    if (!backward)  // which of the two passes runs depends on the output's layout too
        return kHeaderBytes + std::max(simt_segment_bytes(p, 1), p->dtype == HS_BF16 ? segment_bytes(p) : 0);
    return mma_fits(p) ? mma_space(p).total : backward_space(p).total;
}

hs_status heinsen_attention_forward(const heinsen_attention_problem* p, const heinsen_attention_tensor* o, float* state,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    hs_status st = validate(p);
    if (st != HS_OK || nothing(p)) return st;
    if ((st = validate_inputs(p)) != HS_OK) return st;
    if (!o || (p->tokens && !o->ptr)) return HS_ERR_INVALID_ARG;
    if ((st = check_space(p, 0, workspace, workspace_bytes)) != HS_OK) return st;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return p->dtype == HS_F32 ? forward_pass<float>(p, o, state, ws, s) : forward_pass<__nv_bfloat16>(p, o, state, ws, s);
}

hs_status heinsen_attention_backward(const heinsen_attention_problem* p, const heinsen_attention_tensor* d_o,
                                     const float* d_state, void* dq, void* dk, void* dv,
                                     float* dlog_a, float* dstate0, void* workspace, size_t workspace_bytes,
                                     void* stream) {
    hs_status st = validate(p);
    if (st != HS_OK) return st;
    if (nothing(p)) return zero_gradients(p, dq, dk, dv, dlog_a, static_cast<cudaStream_t>(stream));
    if ((st = validate_inputs(p)) != HS_OK) return st;
    if (!d_o || (p->tokens && (!d_o->ptr || !dq || !dk || !dv))) return HS_ERR_INVALID_ARG;
    if (d_state && !std::isfinite(1.0f / p->scale)) return HS_ERR_INVALID_ARG;  // the passes take d_state / scale
    if (mma_fits(p) && ((reinterpret_cast<uintptr_t>(dq) | reinterpret_cast<uintptr_t>(dk) | reinterpret_cast<uintptr_t>(dv)) & 15u))
        return HS_ERR_INVALID_ARG;  // TMA writes them
    if ((st = check_space(p, 1, workspace, workspace_bytes)) != HS_OK) return st;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (mma_fits(p))
        return dlog_a ? mma_backward<true>(p, d_o, d_state, dq, dk, dv, dlog_a, dstate0, ws, s)
                      : mma_backward<false>(p, d_o, d_state, dq, dk, dv, dlog_a, dstate0, ws, s);
    return p->dtype == HS_F32
               ? backward_passes<float>(p, d_o, d_state, dq, dk, dv, dlog_a, dstate0, ws, s)
               : backward_passes<__nv_bfloat16>(p, d_o, d_state, dq, dk, dv, dlog_a, dstate0, ws, s);
}

hs_status heinsen_attention_check(void* stream) {
    int sms, where = 0;
    const hs_status st = hs_internal::current_device(&sms);
    if (st != HS_OK) return st;
    cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaStreamSynchronize", e);
    e = cudaMemcpyFromSymbol(&where, ha::g_gave_up, sizeof where);
    if (e != cudaSuccess) return hs_internal::cuda_fail("cudaMemcpyFromSymbol", e);
    if (!where) return HS_OK;
    const int none = 0;
    e = cudaMemcpyToSymbol(ha::g_gave_up, &none, sizeof none);
    return e == cudaSuccess ? HS_ERR_COPY_TIMEOUT : hs_internal::cuda_fail("cudaMemcpyToSymbol", e);
}

hs_status heinsen_attention_step(const heinsen_attention_problem* p, const heinsen_attention_tensor* o, float* pool_state,
                                 int64_t pool, const int32_t* slots, void* stream) {
    hs_status st = validate(p);
    if (st != HS_OK) return st;
    if (p->tokens != 1 || p->lengths || p->state0 || pool < 0) return HS_ERR_INVALID_ARG;
    if (!slots && pool < p->batch) return HS_ERR_INVALID_ARG;
    if (nothing(p)) return HS_OK;
    if ((st = validate_inputs(p)) != HS_OK) return st;
    if (!o || !o->ptr || (pool && !pool_state)) return HS_ERR_INVALID_ARG;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    ha::Step s;
    s.q = p->q.ptr; s.k = p->k.ptr; s.v = p->v.ptr;
    s.qb = p->q.batch_stride; s.qh = p->q.head_stride; s.qdiv = p->heads / p->q_heads;
    s.kb = p->k.batch_stride; s.kh = p->k.head_stride; s.kdiv = p->heads / p->k_heads;
    s.vb = p->v.batch_stride; s.vh = p->v.head_stride; s.vdiv = p->heads / p->v_heads;
    s.log_a = static_cast<const float*>(p->log_a.ptr); s.ab = p->log_a.batch_stride; s.ah = p->log_a.head_stride;
    s.pool = pool_state; s.slots = slots; s.pool_rows = pool;
    s.heads = p->heads; s.dk = p->k_dim; s.dv = p->v_dim; s.scale = p->scale;
    s.o = const_cast<void*>(o->ptr); s.ob = o->batch_stride; s.oh = o->head_stride;
    cudaStream_t str = static_cast<cudaStream_t>(stream);
    return p->dtype == HS_F32 ? step<float>(s, p->batch, str) : step<__nv_bfloat16>(s, p->batch, str);
}

}  // extern "C"
