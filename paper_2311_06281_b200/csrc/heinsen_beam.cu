// C ABI of beam search: checks of the arguments, workspace layout, launches.
#include "../../include/heinsen_beam.h"

#include <cstring>

#include "ha_host.h"
#include "hb_beam.cuh"

namespace {

using namespace ha_host;

constexpr int kSms = 148;  // B200; sizes workspaces the same wherever they are asked for
constexpr int kMaxBeams = 64;
constexpr long long kMaxVocabulary = (1ll << 31) - (1ll << 20);  // places in a row are 32 bits, past the end of its last part too

hs_status validate(const heinsen_beam_problem* p) {
    if (!p || p->batch < 0 || p->vocabulary < 1 || p->vocabulary > kMaxVocabulary) return HS_ERR_INVALID_ARG;
    if (p->beams < 1 || p->beams > kMaxBeams || p->keep < 1 || p->keep > hb::kMaxKeep) return HS_ERR_INVALID_ARG;
    if (p->keep > p->beams * p->vocabulary) return HS_ERR_INVALID_ARG;
    if (p->dtype != HS_F32 && p->dtype != HS_BF16) return HS_ERR_INVALID_ARG;
    if (p->ended && (p->end_token < 0 || p->end_token >= p->vocabulary)) return HS_ERR_INVALID_ARG;
    if (p->batch > 0x7fffffffll / p->beams) return HS_ERR_INVALID_ARG;
    return HS_OK;
}

// Logits of a thread: 32 of them (8192 a CTA), or 8 where that would leave an SM in two without a CTA.  Both kernels together, with 8
// and with 32 (bf16, keep 4 to 8): 16 CTAs of 8192 logits 8.5 us, 10.2 us (4 rows; 2 rows 10.9, 10.6); 64 of them 11.2, 11.1; 128 of
// them 12.0, 11.1 (4 rows: 17.7, 11.7); 256 of them 14.6, 11.6; 1024 of them 26.2, 18.0.
int per_thread(const heinsen_beam_problem* p) { return p->batch * p->beams * ((p->vocabulary + 8191) / 8192) > kSms / 2 ? 32 : 8; }
long long parts_of(const heinsen_beam_problem* p) {
    const long long each = hb::kThreads * per_thread(p);
    return (p->vocabulary + each - 1) / each;
}
// Does every row begin at an address of 16 bytes?
bool whole_rows(const heinsen_beam_problem* p) {
    const long long vec = p->dtype == HS_F32 ? 4 : 8;
    return (reinterpret_cast<uintptr_t>(p->logits) & 15u) == 0 && (p->batch == 1 || p->batch_stride % vec == 0) && (p->beams == 1 || p->beam_stride % vec == 0);
}

struct Space {
    size_t tokens, sums, total;
};
Space space_of(const heinsen_beam_problem* p) {
    const size_t rows = (size_t)p->batch * p->beams * parts_of(p);
    Space s;
    s.tokens = up256(rows * p->keep * 4);
    s.sums = s.tokens + up256(rows * p->keep * 4);
    s.total = s.sums + up256(rows * sizeof(double2)) + 256;
    return s;
}

template <class T> hs_status select(const heinsen_beam_problem* p, const hb::Select& s, cudaStream_t stream) {
    const long long grid = p->batch * p->beams * s.parts;
    if (grid > 0x7fffffffll) return HS_ERR_INVALID_ARG;
    auto go = [&](auto fn) { fn<<<(unsigned)grid, hb::kThreads, 0, stream>>>(s); };
    const bool whole = whole_rows(p);
    if (per_thread(p) == 32) go(whole ? hb::part_kernel<T, 32, true> : hb::part_kernel<T, 32, false>);
    else go(whole ? hb::part_kernel<T, 8, true> : hb::part_kernel<T, 8, false>);
    const hs_status st = launched("part_kernel");
    if (st != HS_OK) return st;
    hb::join_kernel<<<(unsigned)p->batch, hb::kThreads, 0, stream>>>(s);
    return launched("join_kernel");
}

template <class Unit> hs_status reorder(hb::Reorder r, long long batch, cudaStream_t stream) {
    const long long tiles = (r.row_bytes + (long long)sizeof(Unit) * hb::kThreads - 1) / ((long long)sizeof(Unit) * hb::kThreads);
    if (tiles > 0x7fffffffll / batch) return HS_ERR_INVALID_ARG;
    r.tiles = (int)tiles;
    const unsigned grid = (unsigned)(batch * tiles);
    if (r.beams <= 4) hb::reorder_kernel<Unit, 4><<<grid, hb::kThreads, 0, stream>>>(r);
    else if (r.beams <= 8) hb::reorder_kernel<Unit, 8><<<grid, hb::kThreads, 0, stream>>>(r);
    else if (r.beams <= 16) hb::reorder_kernel<Unit, 16><<<grid, hb::kThreads, 0, stream>>>(r);
    else if (r.beams <= 32) hb::reorder_kernel<Unit, 32><<<grid, hb::kThreads, 0, stream>>>(r);
    else if constexpr (sizeof(Unit) <= 8) hb::reorder_kernel<Unit, 64><<<grid, hb::kThreads, 0, stream>>>(r);
    return launched("reorder_kernel");
}

}  // namespace

extern "C" {

size_t heinsen_beam_workspace_bytes(const heinsen_beam_problem* p) { return validate(p) == HS_OK ? space_of(p).total : 0; }

hs_status heinsen_beam_select(const heinsen_beam_problem* p, float* out_scores, int32_t* out_parents, int32_t* out_tokens, void* workspace,
                              size_t workspace_bytes, void* stream) {
    hs_status st = validate(p);
    if (st != HS_OK || p->batch == 0) return st;
    if (!p->logits || !p->scores || !out_scores || !out_parents || !out_tokens) return HS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->logits) % (p->dtype == HS_F32 ? 4 : 2)) return HS_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HS_ERR_INVALID_ARG;
    const Space sp = space_of(p);
    if (workspace_bytes < sp.total) return HS_ERR_WORKSPACE_TOO_SMALL;
    int sms;
    if ((st = hs_internal::current_device(&sms)) != HS_OK) return st;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    hb::Select s;
    s.logits = p->logits; s.sb = p->batch_stride; s.sw = p->beam_stride;
    s.vocabulary = p->vocabulary;
    s.beams = p->beams; s.keep = p->keep; s.parts = (int)parts_of(p);
    s.scores = p->scores; s.ended = p->ended; s.end_token = p->end_token;
    s.part_value = reinterpret_cast<float*>(ws);
    s.part_token = reinterpret_cast<int*>(ws + sp.tokens);
    s.part_sum = reinterpret_cast<double2*>(ws + sp.sums);
    s.out_scores = out_scores; s.out_parents = out_parents; s.out_tokens = out_tokens;
    cudaStream_t str = static_cast<cudaStream_t>(stream);
    return p->dtype == HS_F32 ? select<float>(p, s, str) : select<__nv_bfloat16>(p, s, str);
}

hs_status heinsen_beam_reorder(void* state, int64_t pool, int64_t row_bytes, const int32_t* parents, const int32_t* slots, int64_t batch,
                               int32_t beams, void* stream) {
    if (pool < 0 || row_bytes < 0 || batch < 0 || beams < 1 || beams > kMaxBeams || batch > 0x7fffffffll / beams) return HS_ERR_INVALID_ARG;
    if (pool && row_bytes > (1ll << 62) / pool) return HS_ERR_INVALID_ARG;
    if (!slots && pool < batch * beams) return HS_ERR_INVALID_ARG;
    if (batch == 0 || pool == 0 || row_bytes == 0) return HS_OK;
    if (!state || !parents) return HS_ERR_INVALID_ARG;
    int sms;
    const hs_status st = hs_internal::current_device(&sms);
    if (st != HS_OK) return st;
    const hb::Reorder r{static_cast<uint8_t*>(state), pool, row_bytes, parents, slots, beams, 0};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uintptr_t fit = reinterpret_cast<uintptr_t>(state) | (uintptr_t)row_bytes;
    // units of 16 bytes, of which a thread can hold 32; of 8 for more beams or where rows do not begin at such addresses
    if (fit % 16 == 0 && beams <= 32) return reorder<uint4>(r, batch, s);
    if (fit % 8 == 0) return reorder<uint2>(r, batch, s);
    if (fit % 4 == 0) return reorder<uint32_t>(r, batch, s);
    return reorder<uint8_t>(r, batch, s);
}

}  // extern "C"
