// Beam search: the best continuations of a group of beams, and the states that follow them.
//
// Within a beam the candidates' order is that of its logits, so a row of logits is read once: a CTA has a part of a row in
// registers, forms its largest value, the sum of the exponentials over that, and its `keep` largest logits; a CTA for each group
// joins the parts' sums to the beams' log-sums and picks from the parts' lists.  Bound by reading the logits.
#pragma once
#include "ha_common.cuh"

namespace hb {

constexpr int kThreads = 256;
constexpr int kMaxKeep = 64;
constexpr int kList = 256;  // candidates of a part that are sorted at once

struct Select {
    const void* logits;
    long long sb, sw;  // strides of batch and beam
    long long vocabulary;
    int beams, keep, parts;
    const float* scores;
    const uint8_t* ended;
    long long end_token;
    float* part_value;   // [rows][parts][keep]
    int* part_token;
    double2* part_sum;   // [rows][parts]: largest value, sum of the exponentials
    float* out_scores;
    int *out_parents, *out_tokens;
};

// Numbers in the order of their size as unsigned ones; both zeros are one
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// Bound by HBM and by the instructions for a logit (an exponential and a test): 256 rows of 100003 float32 logits, a fifth of them of
// ended beams, 28 us for 82 MB; 8 logits a thread where there are few rows (4 rows of 32000 bf16: 3.3 us).
// Parts of many tiles of 16 logits a thread, the next one's loads ahead, gave the part 31 to 38 us and the join 7.3: no gain.
// One part of one row; kPer logits a thread.  Which of a row's logits a thread has is the same for all rows of a call, wherever they
// begin, so that beams with the same logits have the same sums to the last bit and their candidates come in the order of the beams.
// kWhole: every row begins at an address of 16 bytes, and a thread has vectors of as many; else single logits, a warp's side by side.
template <class T, int kPer, bool kWhole>
__global__ void __launch_bounds__(kThreads, kPer == 32 ? 4 : 6) part_kernel(const Select p) {
    constexpr int kVec = kWhole ? 16 / sizeof(T) : 1, kVecs = kPer / kVec;
    __shared__ float red_max[kThreads / 32];
    __shared__ double red_sum[kThreads / 32];
    __shared__ __align__(16) uint32_t tops[kThreads];
    __shared__ uint32_t least;
    __shared__ uint32_t list_key[kList];
    __shared__ int list_token[kList];
    __shared__ int found;
    __shared__ unsigned long long best[kThreads / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int part = blockIdx.x % p.parts;
    const long long row = blockIdx.x / p.parts, b = row / p.beams, w = row % p.beams;
    const T* const from = static_cast<const T*>(p.logits) + b * p.sb + w * p.sw;
    const int first = part * (kThreads * kPer), vocabulary = (int)p.vocabulary;
    if (tid == 0) found = 0;
    if (p.ended && p.ended[row]) return;  // nothing of it is asked for
    float x[kPer];
    auto token = [&](int i) { return first + (i / kVec * kThreads + tid) * kVec + i % kVec; };
    if (first + kThreads * kPer <= vocabulary) {  // all of it is there: no load waits for another's test
        if constexpr (kWhole) {
            uint4 f[kVecs];
#pragma unroll
            for (int u = 0; u < kVecs; ++u) f[u] = __ldcs(reinterpret_cast<const uint4*>(from + token(u * kVec)));
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                const uint32_t r[4] = {f[u].x, f[u].y, f[u].z, f[u].w};
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if constexpr (sizeof(T) == 2) x[u * kVec + i] = __uint_as_float(i & 1 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
                    else x[u * kVec + i] = __uint_as_float(r[i]);
                }
            }
        } else {
            T f[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) f[i] = __ldcs(from + token(i));
#pragma unroll
            for (int i = 0; i < kPer; ++i) x[i] = ha::to_f(f[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int n = token(i);
            x[i] = n < vocabulary ? ha::to_f(from[n]) : __int_as_float(0xff800000);
        }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
    // The keep-th largest of the maxima of disjoint groups (8 lanes each; single threads where more than 16 are asked for) bounds the
    // keep-th best of the part from below, and few logits lie above it.
    const bool few = p.keep <= 16;
    float m = top;
#pragma unroll
    for (int o = 1; o < 8; o *= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if (!few) tops[tid] = ordered(top);
    else if ((lane & 7) == 0) tops[warp * 4 + (lane >> 3)] = ordered(m);
    m = fmaxf(m, __shfl_xor_sync(~0u, m, 8));
    m = fmaxf(m, __shfl_xor_sync(~0u, m, 16));
    if (lane == 0) red_max[warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, red_max[i]);
    float part_sum = 0.0f;  // NaN where a logit is (the maximum passes it over), and for a maximum of +inf, of which m - m is NaN
    if (m == __int_as_float(0xff800000)) {  // none but -inf, and NaN
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (x[i] != x[i]) part_sum = x[i];
    } else {
        // Off by 2^-20 from the 16 roundings of its two chains and their sum, 2^-22 from the exponentials, and 2.3 x 2^-24 from each exponent
        // times its size, 17 in the mean at most for 2^31 logits: less than 2^-18 of the sum.
        const ha::pair minus = ha::make_pair2(-m, -m), base = ha::make_pair2(ha::kLog2e, ha::kLog2e);
        ha::pair sums = 0;
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
            float a, b;
            ha::parts(ha::mul2(ha::add2(ha::make_pair2(x[i], x[i + 1]), minus), base), a, b);
            sums = ha::add2(sums, ha::make_pair2(ha::ex2(a), ha::ex2(b)));
        }
        float a, b;
        ha::parts(sums, a, b);
        part_sum = a + b;
    }
    double sum = (double)part_sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) red_sum[warp] = sum;
    const long long at = row * p.parts + part;
    float* const values = p.part_value + at * p.keep;
    int* const tokens = p.part_token + at * p.keep;
    if (few && warp == 0) {
        const uint32_t own = tops[lane];
        int above = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint32_t other = __shfl_sync(~0u, own, i);
            above += other > own || (other == own && i < lane);
        }
        if (above == p.keep - 1) least = own;
    } else if (!few) {
        const uint32_t own = tops[tid];
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < kThreads; i += 4) {
            const uint4 other = *reinterpret_cast<const uint4*>(tops + i);
            above += (other.x > own || (other.x == own && i < tid)) + (other.y > own || (other.y == own && i + 1 < tid)) +
                     (other.z > own || (other.z == own && i + 2 < tid)) + (other.w > own || (other.w == own && i + 3 < tid));
        }
        if (above == p.keep - 1) least = own;
    }
    __syncthreads();
    if (tid == 0) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) sum += red_sum[i];
        p.part_sum[at] = make_double2((double)m, sum);
    }
    // A bound of -inf (few logits that are not): of those at -inf the first `keep` places are enough.
    const float bound = from_ordered(least), lowest = __int_as_float(0xff800000);
    const int places = bound == lowest ? first + p.keep : vocabulary;
    if (top >= bound)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int n = token(i);
            if (x[i] >= bound && n < (x[i] > lowest ? vocabulary : min(places, vocabulary))) {
                const int to = atomicAdd(&found, 1);
                if (to < kList) {
                    list_key[to] = ordered(x[i]);
                    list_token[to] = (int)n;
                }
            }
        }
    __syncthreads();
    const int count = found;
    if (count <= kList) {  // sorted by value and place: the order in which they came does not matter
        if (tid < count) {
            const uint32_t key = list_key[tid];
            const int n = list_token[tid];
            int rank = 0;
            for (int i = 0; i < count; ++i) rank += list_key[i] > key || (list_key[i] == key && list_token[i] < n);
            if (rank < p.keep) {
                values[rank] = from_ordered(key);
                tokens[rank] = n;
            }
        }
        for (int i = count + tid; i < p.keep; i += kThreads) tokens[i] = -1;  // the part holds fewer
    } else {  // many equal ones
        // one after the other: the best of those that come after the last one in the order (value, then place)
        unsigned long long last = ~0ull;
        for (int k = 0; k < p.keep; ++k) {
            unsigned long long mine = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int n = token(i);
                const unsigned long long key = (unsigned long long)ordered(x[i]) << 32 | (uint32_t)~(uint32_t)n;
                if (n < vocabulary && key < last && key > mine) mine = key;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const unsigned long long other = __shfl_xor_sync(~0u, mine, o);
                mine = other > mine ? other : mine;
            }
            __syncthreads();
            if (lane == 0) best[warp] = mine;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kThreads / 32; ++i) mine = best[i] > mine ? best[i] : mine;
            last = mine;
            if (tid == 0) {
                values[k] = from_ordered((uint32_t)(mine >> 32));
                tokens[k] = mine ? (int)~(uint32_t)mine : -1;
            }
            if (!mine) last = 0;
        }
    }
}

// A candidate: its value, its logit, and beam and token as one number.
struct Candidate {
    double value;
    float logit;
    long long place;
};
// The order of candidates.  Equal values come by beam; those of one beam by logit, since two logits can have the same sum with a large
// score or log-sum in 64 bits, and the parts' lists, of which no more than `keep` are at hand, are in the logits' order.
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {  // no branches: loads of more than one go together
    const bool by_place = ((int)(a.place >> 32) != (int)(b.place >> 32)) | (a.logit == b.logit);
    return (a.value > b.value) | ((a.value == b.value) & ((by_place & (a.place < b.place)) | (!by_place & (a.logit > b.logit))));
}
__device__ __forceinline__ Candidate across(const Candidate& c, int lanes) {
    return {__shfl_xor_sync(~0u, c.value, lanes), __shfl_xor_sync(~0u, c.logit, lanes), __shfl_xor_sync(~0u, c.place, lanes)};
}

// The best of a group.  Candidates are formed in 64 bits; as above, the keep-th best of the threads' own best bounds the keep-th best
// of all, and those above it are sorted.
// Bound by latency, a CTA for a group: 8 beams of 13 parts with 8 candidates each 8.5 us (11 us with one load of a lane at a time),
// 4 beams of 16 parts with 4 each 5.1 us.  Comparisons with branches in them: 15 us and 8 us.
constexpr int kJoinList = 512;
__global__ void __launch_bounds__(kThreads) join_kernel(const Select p) {
    __shared__ double logs[64];
    __shared__ int state[64];  // 0: as its logits say; 1: ended; 2: out
    __shared__ double value_of[kJoinList];
    __shared__ long long place_of[kJoinList];
    __shared__ float logit_of[kJoinList];
    __shared__ double least_value;
    __shared__ long long least_place;
    __shared__ float least_logit;
    __shared__ int found;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long b = blockIdx.x;
    const double lowest = -__longlong_as_double(0x7ff0000000000000ll);
    const Candidate none{lowest, 0.0f, 0x7fffffffffffffffll};
    if (tid == 0) found = 0;
    for (int w = warp; w < p.beams; w += kThreads / 32) {
        const long long row = b * p.beams + w;
        const float score = p.scores[row];
        const bool ended = p.ended && p.ended[row];
        double m = lowest, s = 0.0;
        if (!ended) {
            for (int i = lane; i < p.parts; i += 32) m = fmax(m, p.part_sum[row * p.parts + i].x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(~0u, m, o));
            for (int i = lane; i < p.parts; i += 32) {
                const double2 f = p.part_sum[row * p.parts + i];
                s += f.x == m || f.x == lowest ? f.y : f.y * exp(f.x - m);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        }
        const double l = m + log(s);
        if (lane == 0) {
            logs[w] = (double)score - l;
            state[w] = !isfinite(score) ? 2 : ended ? 1 : isfinite(l) ? 0 : 2;
        }
    }
    __syncthreads();
    const int lists = p.parts * p.keep;
    // Of a beam without candidates of its own the first tokens count, at -inf, as many as could be needed.
    auto each_candidate = [&](auto take) {
        for (int w = warp; w < p.beams; w += kThreads / 32) {
            const int how = state[w];
            const long long row0 = (long long)w << 32;
            if (how == 0) {
                const double base = logs[w];
                const long long at = (b * p.beams + w) * lists;
                for (int i = lane; i < lists; i += 128) {  // four of a lane's loads together
                    int n[4];
                    float v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const bool on = i + 32 * u < lists;
                        n[u] = on ? p.part_token[at + i + 32 * u] : -1;
                        v[u] = on ? p.part_value[at + i + 32 * u] : 0.0f;  // (that of no token is never used)
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (n[u] >= 0) take(Candidate{base + (double)v[u], v[u], row0 + n[u]});
                }
            } else {
                for (int i = lane; i <= p.keep && i < p.vocabulary; i += 32)
                    if (!(how == 1 && i == p.end_token)) take(Candidate{lowest, 0.0f, row0 + i});
                if (how == 1 && lane == 0) take(Candidate{(double)p.scores[b * p.beams + w], 0.0f, row0 + p.end_token});
            }
        }
    };
    auto put = [&](int at, const Candidate& c) {
        value_of[at] = c.value;
        logit_of[at] = c.logit;
        place_of[at] = c.place;
    };
    auto get = [&](int at) { return Candidate{value_of[at], logit_of[at], place_of[at]}; };
    Candidate own = none;
    each_candidate([&](const Candidate& c) {
        if (before(c, own)) own = c;
    });
    const bool few = p.keep <= 16;
    if (few)  // the best of every eight threads
#pragma unroll
        for (int o = 1; o < 8; o *= 2) {
            const Candidate c = across(own, o);
            if (before(c, own)) own = c;
        }
    const int each = few ? 8 : 1, members = kThreads / each;
    if (tid % each == 0) put(tid / each, own);
    __syncthreads();
    if (tid < members) {
        own = get(tid);
        int rank = 0;
#pragma unroll 4
        for (int i = 0; i < members; ++i) {
            const Candidate c = get(i);
            rank += before(c, own) | ((c.place == own.place) & (i < tid));
        }
        if (rank == p.keep - 1) {
            least_value = own.value;
            least_logit = own.logit;
            least_place = own.place;
        }
    }
    __syncthreads();
    const Candidate bound{least_value, least_logit, least_place};
    each_candidate([&](const Candidate& c) {
        if (!before(bound, c)) {
            const int to = atomicAdd(&found, 1);
            if (to < kJoinList) put(to, c);
        }
    });
    __syncthreads();
    const int count = found;
    auto choose = [&](int k, const Candidate& c) {
        const long long to = b * p.keep + k;
        p.out_scores[to] = (float)c.value;
        p.out_parents[to] = (int)(c.place >> 32);
        p.out_tokens[to] = (int)c.place;
    };
    if (count <= kJoinList) {
        for (int at = tid; at < count; at += kThreads) {
            const Candidate c = get(at);
            int r = 0;
            for (int i = 0; i < count; ++i) r += before(get(i), c);
            if (r < p.keep) choose(r, c);
        }
        return;
    }
    // More than the list holds, one after the other: where a few threads have very many of the best, or where fewer threads than `keep` asks
    // for have any (few beams: a beam is one warp's), so that nothing bounds them.
    Candidate last{-lowest, 0.0f, -1};
    for (int k = 0; k < p.keep; ++k) {
        own = none;
        each_candidate([&](const Candidate& c) {
            if (before(last, c) && before(c, own)) own = c;
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const Candidate c = across(own, o);
            if (before(c, own)) own = c;
        }
        __syncthreads();
        if (lane == 0) put(warp, own);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i)
            if (before(get(i), own)) own = get(i);
        last = own;
        if (tid == 0) choose(k, own);
    }
}

// ---------------------------------------------------------------------------------------------------------------- states

struct Reorder {
    uint8_t* state;
    long long pool, row_bytes;
    const int *parents, *slots;
    int beams, tiles;
};

// A CTA has a piece of the rows of one group: every thread reads its unit of all rows that move before it writes any.  Bound by
// the two trips of the rows that move: 48 groups of four beams with 1 MB each, of which
// three in four move (120 MB read, 151 written), 47 us.
template <class Unit, int kBeams>
__global__ void __launch_bounds__(kThreads) reorder_kernel(const Reorder p) {
    __shared__ long long from[kBeams], to[kBeams];
    const int tid = threadIdx.x, tile = blockIdx.x % p.tiles;
    const long long b = blockIdx.x / p.tiles;
    if (tid < kBeams) {
        long long source = -1, target = -1;
        if (tid < p.beams) {
            auto slot = [&](int w) {
                const long long s = p.slots ? (long long)p.slots[b * p.beams + w] : b * p.beams + w;
                return s < 0 || s >= p.pool ? -1 : s;
            };
            const int parent = p.parents[b * p.beams + tid];
            if (parent >= 0 && parent < p.beams) {
                source = slot(parent);
                target = slot(tid);
            }
            if (source < 0 || target < 0 || source == target) source = target = -1;
        }
        from[tid] = source < 0 ? -1 : source * p.row_bytes;
        to[tid] = target * p.row_bytes;
    }
    __syncthreads();
    const long long at = ((long long)tile * kThreads + tid) * sizeof(Unit);
    if (at >= p.row_bytes) return;
    Unit held[kBeams];
#pragma unroll
    for (int w = 0; w < kBeams; ++w)
        if (from[w] >= 0) held[w] = *reinterpret_cast<const Unit*>(p.state + from[w] + at);
#pragma unroll
    for (int w = 0; w < kBeams; ++w)
        if (from[w] >= 0) *reinterpret_cast<Unit*>(p.state + to[w] + at) = held[w];
}

}  // namespace hb
