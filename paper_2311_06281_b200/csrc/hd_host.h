// What the forward and the backward pass of the delta rule share on the host.
#pragma once
#include <cstring>

#include "../../include/heinsen_delta.h"
#include "ha_host.h"
#include "hd_scan_mma.cuh"

namespace hd_host {

using namespace ha_host;

#pragma GCC visibility push(hidden)
// The word of the current device that says where a bounded wait of any call ran out; NULL where CUDA fails.
int* gave_up_word();
size_t backward_bytes(const heinsen_delta_problem* p);
#pragma GCC visibility pop

constexpr int kSms = 148;  // B200; sizes the grid and workspaces the same wherever they are asked for

inline int width_of(int dk) { return dk <= 64 ? 64 : dk <= 128 ? 128 : 256; }

struct View {  // one [batch, tokens, heads', dim] tensor
    Rows rows;
    int own_heads, dim;
};
inline View view_of(const heinsen_attention_tensor& t, int heads, int own, int dim) { return {rows_of(t, heads, own), own, dim}; }

// Can TMA address it?  bf16, 16-byte base and strides; a stride of a dimension of one is never used.
inline bool tma_strides(const View& v, long long batch, long long tokens) {
    const long long s[3] = {v.own_heads > 1 ? v.rows.sh : 8, tokens > 1 ? v.rows.st : 8, batch > 1 ? v.rows.sb : 8};
    for (long long x : s)
        if (x <= 0 || x % 8 || x >= (1ll << 38)) return false;
    return v.dim % 8 == 0 && (reinterpret_cast<uintptr_t>(v.rows.ptr) & 15u) == 0;
}
inline bool encode(CUtensorMap* m, const View& v, long long batch, long long tokens, int columns, int rows) {
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)v.dim, (cuuint64_t)v.own_heads, (cuuint64_t)tokens, (cuuint64_t)batch};
    const cuuint64_t any = 256;
    const cuuint64_t strides[3] = {v.own_heads > 1 ? (cuuint64_t)v.rows.sh * 2 : any, tokens > 1 ? (cuuint64_t)v.rows.st * 2 : any,
                                   batch > 1 ? (cuuint64_t)v.rows.sb * 2 : any};
    const cuuint32_t box[4] = {(cuuint32_t)columns, 1, (cuuint32_t)rows, 1}, one[4] = {1, 1, 1, 1};
    for (int again = 0;; ++again) {
        const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(v.rows.ptr), dims, strides, box, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, columns == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_32B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r == CUDA_SUCCESS || again) return r == CUDA_SUCCESS;
        cudaFree(nullptr);  // a thread that has made no runtime call yet has no context for the driver's
    }
}

// Bytes of a tensor laid out as bf16 terms for TMA; 0 where it is loaded as it is.
inline size_t terms_bytes(const heinsen_attention_problem* p, const View& v) {
    if (p->tokens == 0 || (p->dtype == HS_BF16 && tma_strides(v, p->batch, p->tokens))) return 0;
    return up256((size_t)(p->dtype == HS_F32 ? 3 : 1) * p->batch * p->tokens * v.own_heads * ((v.dim + 7) / 8 * 8) * 2);
}
// The tensor map of a tensor; where it has to be laid out anew, that of the place in `space` which `all` then says it goes to.
template <class T, int TI>
hs_status map_of(CUtensorMap* m, const heinsen_attention_problem* p, const View& v, uint8_t* space, int columns, int rows, hd::Terms* all) {
    View w = v;
    if (terms_bytes(p, v)) {
        const int width = (v.dim + 7) / 8 * 8;
        const long long sh = width, stk = sh * v.own_heads;
        const bool whole = v.dim % 8 == 0 && (v.rows.sb | v.rows.st | v.rows.sh) % 4 == 0 && (reinterpret_cast<uintptr_t>(v.rows.ptr) & 15u) == 0;
        all->tokens = (uint32_t)p->tokens;
        all->tensors[all->count++] = {v.rows, reinterpret_cast<__nv_bfloat16*>(space), p->batch * p->tokens * v.own_heads * (width / 8), (uint32_t)v.own_heads,
                                      v.dim, width, whole};
        w = {{space, stk * p->tokens, stk, sh, 1}, v.own_heads, width};
    }
    if (!encode(m, w, p->batch * TI, p->tokens, columns, rows)) return hs_internal::cuda_fail("cuTensorMapEncodeTiled", cudaErrorInvalidValue);
    return HS_OK;
}
template <class T, int TI> hs_status launch_terms(const hd::Terms& all, cudaStream_t stream) {
    if (!all.count) return HS_OK;
    long long most = 0;
    for (int i = 0; i < all.count; ++i) most = std::max(most, all.tensors[i].pieces);
    const dim3 grid((unsigned)std::min<long long>((most + 255) / 256, kSms * 16), all.count);
    hd::terms_kernel<TI, T><<<grid, 256, 0, stream>>>(all);
    return launched("terms_kernel");
}

inline hd::Params params_of(const heinsen_delta_problem* dp, int chunk, uint8_t* ws) {
    const heinsen_attention_problem* p = &dp->a;
    hd::Params q;
    std::memset(&q, 0, sizeof q);
    q.log_a = static_cast<const float*>(p->log_a.ptr);
    q.ab = p->log_a.batch_stride; q.at = p->log_a.token_stride; q.ah = p->log_a.head_stride;
    q.beta = static_cast<const float*>(dp->beta.ptr);
    q.bb = dp->beta.batch_stride; q.bt = dp->beta.token_stride; q.bh = dp->beta.head_stride;
    q.lengths = p->lengths;
    q.batch = (int)p->batch; q.tokens = (int)p->tokens; q.heads = p->heads;
    q.chunks = (int)((p->tokens + chunk - 1) / chunk);
    q.qdiv = p->heads / p->q_heads; q.kdiv = p->heads / p->k_heads; q.vdiv = p->heads / p->v_heads;
    q.dk = p->k_dim; q.dv = p->v_dim;
    q.scale = p->scale;
    q.fault = reinterpret_cast<ha::Fault*>(ws);
    q.call_id = hs_internal::call_id();
    q.spin = hs_internal::spin_limit();
    q.mute = (int)std::min<long long>(hs_internal::mute_tile(), 0x7fffffff);
    return q;
}

inline long long chunks_of(const heinsen_attention_problem* p) {
    const int c = hd::chunk_tokens(width_of(p->k_dim));
    return p->batch * p->heads * ((p->tokens + c - 1) / c);
}
template <int C, int TM, int TP, bool kBack> size_t image_bytes(const heinsen_attention_problem* p) { return up256((size_t)chunks_of(p) * hd::Image<C, TM, TP, kBack>::end); }

// Slices of sixteen columns of V that a CTA of the mma.sync scans has: two where there would be more CTAs than SMs otherwise, since a
// chunk of two at once takes 3.4 us and two CTAs of one slice one after the other 4.8 (keys 128 wide, one CTA to an SM).
inline int slices_for(long long pairs, int slices) { return pairs * slices > kSms && slices > 1 ? hd::kMaxSlices : 1; }

template <int KP, int C, int TI, int TM, int TP, bool kBack>
hs_status launch_chunks(const CUtensorMap& mq, const CUtensorMap& mk, const hd::Params& q, int* word, cudaStream_t stream) {
    using L = hd::ChunkLayout<KP, C, TI, TM, TP, kBack>;
    const auto fn = hd::chunk_kernel<KP, C, TI, TM, TP, kBack>;
    static std::atomic<unsigned long long> done{0};
    const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)L::end, done);
    if (st != HS_OK) return st;
    fn<<<(unsigned)((long long)q.batch * q.heads * q.chunks), 2 * C, L::end, stream>>>(mq, mk, q, word);
    return launched("chunk_kernel");
}

template <class L, class Fn>
hs_status launch_slices(Fn fn, std::atomic<unsigned long long>& done, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const hd::Params& q,
                        int* word, cudaStream_t stream) {
    static_assert(L::end(hd::kMaxSlices) <= 232448, "shared memory");
    const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)L::end(hd::kMaxSlices), done);
    if (st != HS_OK) return st;
    const long long pairs = (long long)q.batch * q.heads;
    const int slices = (q.dv + 15) / 16, each = slices_for(pairs, slices);
    const long long grid = pairs * ((slices + each - 1) / each);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    hd::Params w = q;
    w.slices = each;
    fn<<<(unsigned)grid, 128 * (each + 1), L::end(each), stream>>>(mq, mk, mv, w, word);
    return launched("scan_kernel");
}
template <int KP, int C, int TI, int TM, int TP, bool kOut, class T>
hs_status launch_scan(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const hd::Params& q, int* word, cudaStream_t stream) {
    static std::atomic<unsigned long long> done{0};
    return launch_slices<hd::ScanLayout<KP, C, TI, TM, TP, kOut, !kOut>>(hd::scan_kernel<KP, C, TI, TM, TP, kOut, T>, done, mq, mk, mv, q, word, stream);
}

// Whether the passes can run on tcgen05: bf16 and keys up to 128 wide; and whether they do.
template <int KP, int TI> constexpr bool fits_tcgen05() { return TI == 1 && KP <= 128; }

// Which of the two: a CTA with four warps for each of one or two slices of sixteen columns of V (mma.sync), or one with 128 columns
// (tcgen05).  Measured for a chunk, keys and values 128 wide, with one CTA to an SM: one slice 2.4 us, two 3.4 us, 128 columns 5.4 us
// forward; for the gradients (both passes) two slices 6.7 us, 128 columns 13.7 us.  So two slices as long as their waves over the SMs
// are at most 3/2 (2) of the other's.  Sequences of 1024 tokens, mma.sync and tcgen05 forward, and both passes for the gradients, us:
//   keys, values 128, 128: 32 pairs 56, 86; 110, 221.  64 pairs 110, 93; 215, 220.  80 pairs 161, 94; 315, 223.  160 pairs 266, 183; 526, 431.
//   64, 64: 64 pairs 48, 68; 93, 155.  80 pairs 92, 69; 176, 157.  128 pairs 94, 76; 178, 176.  160 pairs 137, 137; 261, 298.
//   64, 128: 64 pairs 94, 67; 179, 162.    128, 64: 64 pairs 56, 90; 110, 197.  80 pairs 107, 93; 211, 198.
// Where it takes the slower one (64, 64, 80 pairs; 64, 128, 64 pairs, gradients) that costs 12% at most.
inline bool many_slices(const heinsen_attention_problem* p, bool backward) {
    const long long pairs = p->batch * p->heads, slices = (p->v_dim + 15) / 16, two = (pairs * ((slices + 1) / 2) + kSms - 1) / kSms,
                    all = (pairs * ((p->v_dim + 127) / 128) + kSms - 1) / kSms;
    return pairs * slices > kSms && (backward ? two > 2 * all : 2 * two > 3 * all);
}

template <int KP, int kMode, class T>
hs_status launch_pass(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const hd::Params& q, int* word, cudaStream_t stream) {
    using L = hd::PassLayout<KP, kMode>;
    static_assert(L::end <= 232448, "shared memory");
    const auto fn = hd::pass_kernel<KP, kMode, T>;
    static std::atomic<unsigned long long> done{0};
    const hs_status st = allow_smem(reinterpret_cast<const void*>(fn), (int)L::end, done);
    if (st != HS_OK) return st;
    const long long grid = (long long)q.batch * q.heads * ((q.dv + 127) / 128);
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    fn<<<(unsigned)grid, hd::kPassThreads, L::end, stream>>>(mq, mk, mv, q, word);
    return launched("pass_kernel");
}

}  // namespace hd_host
