// Log probabilities of the drafted tokens under the rows that predict them, with each row's log-sum-exp, entropy and most likely tokens.
//
// One pass over the logits, in two kernels:
//   logprob_scan_kernel   a warp takes a (row, vocabulary chunk) item, 32 logits per lane and round, the next round's loads in
//                         flight meanwhile.  Per lane m = running maximum, s = sum e^(x - m), t = sum e^(x - m) (x - m);
//                         per warp the chunk's best tokens, one per lane, sorted.
//   logprob_merge_kernel  a CTA per row joins the chunks:  lse = m + ln s,  entropy = ln s - t / s,  and scores a token.
// Bound by the logits' bytes: per element a maximum, a subtraction, a product, a clamp, an ex2 and two sums.
// The list costs little because it is looked at only in rounds with a logit above its last entry: in the first round that limit is
// taken from the lanes' maxima (at least `top` logits are not below the top-th largest of them), later it only rises.
#pragma once

#include "accept.cuh"
#include "owl_common.cuh"

namespace owl {

constexpr int kMaxTop = 32;              // alternatives per row: one per lane
constexpr int kScoreWarps = 8;
constexpr int kScoreRound = 1024;        // logits per warp and round
constexpr int kScoreMaxChunk = 16384;
constexpr int kScoreCtasPerSm = 2;

struct ScorePartial { float m, s, t, pad; };

struct ScoreParams {
    const void* logits;                  // [N, V] fp32, bf16 or fp16
    const int32_t* tokens;               // [N]
    const int32_t* node_offsets;         // may be null: uniform
    const int32_t* tree_parent;          // null: token n is scored on row n
    float* logprob;                      // each of the outputs may be null
    float* entropy;
    float* lse;
    int32_t* top_ids;                    // [N, top]
    float* top_logprobs;
    ScorePartial* part;                  // [N, chunks]
    unsigned long long* part_keys;       // [N, chunks, top], descending
    float2* row_sums;                    // [N] a row's (m, s), for the rows of later launches of the call; null: there are none
    int32_t* status;
    int32_t batch, total_nodes, nodes_uniform, max_nodes, vocab, top, chunk, chunks;
    int32_t row0, rows;                  // this launch's rows [row0, row0 + rows); the partials are counted from row0
};

// What an entry of the list is ordered by: larger logit first, then the lower token.  0: no entry (-inf and NaN make none).
__device__ __forceinline__ unsigned long long score_key(float x, uint32_t idx) { return x > -INFINITY ? argmax_key(x, idx) : 0ull; }
__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ unsigned long long shfl_key(unsigned long long k, int lane) { return __shfl_sync(0xffffffffu, k, lane); }

// Two descending lists of 32 (one entry per lane) to the descending list of the 32 largest: the larger of a[i] and b[31 - i] are
// those, in a bitonic order, which five exchanges sort.
__device__ __forceinline__ unsigned long long merge_lists(unsigned long long a, unsigned long long b) {
    const int lane = threadIdx.x & 31;
    const unsigned long long r = shfl_key(b, 31 - lane);
    a = a > r ? a : r;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, a, o);
        const bool larger = (lane & o) == 0;
        a = (other > a) == larger ? other : a;
    }
    return a;
}
// One key per lane, in any order, to a descending list (bitonic sort).
__device__ __forceinline__ unsigned long long sort_list(unsigned long long a) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int o = size >> 1; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, a, o);
            const bool larger = ((lane & o) == 0) == ((lane & size) == 0);
            a = (other > a) == larger ? other : a;
        }
    return a;
}
// `mine`: a candidate per lane, 0 for none.  A few go in one by one, more are sorted and merged.
__device__ __forceinline__ unsigned long long join_list(unsigned long long list, unsigned long long mine) {
    const int lane = threadIdx.x & 31;
    unsigned from = __ballot_sync(0xffffffffu, mine != 0ull);
    if (__popc(from) > 6) return merge_lists(list, sort_list(mine));
    while (from) {
        const unsigned long long k = shfl_key(mine, __ffs(from) - 1);
        from &= from - 1;
        const int at = __popc(__ballot_sync(0xffffffffu, list > k));
        const unsigned long long up = __shfl_up_sync(0xffffffffu, list, 1);
        list = lane < at ? list : lane == at ? k : up;
    }
    return list;
}

__device__ __forceinline__ float exp_of(float d) { return fast_exp2(d * 1.4426950408889634f); }

// (m, s, t) of two sets of logits joined; a set without a finite logit has m = -inf and zeros.
__device__ __forceinline__ void join_sums(float& m, float& s, float& t, float m2, float s2, float t2) {
    const float mm = fmaxf(m, m2);
    const float d1 = m == mm ? 0.f : m - mm, d2 = m2 == mm ? 0.f : m2 - mm;      // (infinities of one sign differ by nothing)
    const float a1 = exp_of(d1), a2 = exp_of(d2);
    // t is measured from m: moving the reference adds d s; a set that weighs nothing adds nothing
    t = (a1 > 0.f ? a1 * fmaf(d1, s, t) : 0.f) + (a2 > 0.f ? a2 * fmaf(d2, s2, t2) : 0.f);
    s = a1 * s + a2 * s2;
    m = mm;
}

// One lane's 32 logits of a round (kWide: 4-byte elements, four per load; else eight).
template <typename T> struct ScoreLoad {
    static constexpr int kPer = 16 / (int)sizeof(T), kLoads = 32 / kPer;
    uint4 u[kLoads];
};
__device__ __forceinline__ uint4 ld_stream_u4(const uint4* ptr, uint64_t policy) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(ptr), "l"(policy));
    return v;
}
__device__ __forceinline__ float score_of(float x) { return x; }
__device__ __forceinline__ float score_of(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float score_of(__half x) { return __half2float(x); }
__device__ __forceinline__ void score_unpack(const ScoreLoad<float>& l, float (&x)[32]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[4 * j] = __uint_as_float(l.u[j].x); x[4 * j + 1] = __uint_as_float(l.u[j].y);
        x[4 * j + 2] = __uint_as_float(l.u[j].z); x[4 * j + 3] = __uint_as_float(l.u[j].w);
    }
}
template <typename T>
__device__ __forceinline__ void score_unpack(const ScoreLoad<T>& l, float (&x)[32]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w[4] = {l.u[j].x, l.u[j].y, l.u[j].z, l.u[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(T) == 2 && std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[8 * j + 2 * i] = f.x; x[8 * j + 2 * i + 1] = f.y;
            } else {
                x[8 * j + 2 * i] = __uint_as_float(w[i] << 16); x[8 * j + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
}

// A lane's sums and the warp's list while it works through a chunk.
struct ScoreState {
    float m = -INFINITY, s = 0.f, t = 0.f;
    unsigned long long list = 0ull;
    float limit = -INFINITY;             // a logit must be above it to enter the list
    bool full = false;                   // the list has `top` entries
};
// The lane's logits of a round (absent ones: -inf).
template <int kCount>
__device__ __forceinline__ void score_sums(ScoreState& st, const float (&x)[kCount], float round_max) {
    if (round_max > st.m) {
        if (st.m > -INFINITY) {
            const float d = st.m - round_max, a = exp_of(d);
            st.t = a > 0.f ? a * fmaf(d, st.s, st.t) : 0.f;
            st.s *= a;
        }
        st.m = round_max;
    }
    const float m = st.m;
    float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        // -inf, a NaN, and the NaN of inf - inf all become a difference whose weight is 0
        const float d = fmaxf(x[i] - m, -200.f), e = exp_of(d);
        if (i & 1) { s1 += e; t1 = fmaf(e, d, t1); }
        else { s0 += e; t0 = fmaf(e, d, t0); }
    }
    st.s += s0 + s1;
    st.t += t0 + t1;
}
// Candidates of a round, one per lane at a time.  `at(i)`: the token of the lane's i-th logit; within a lane they ascend, and every
// token of an earlier round is lower than any of this one, so a logit equal to the limit cannot enter.
template <int kCount, typename At>
__device__ __forceinline__ void score_list(ScoreState& st, int top, const float (&x)[kCount], float round_max, At at) {
    constexpr unsigned kAll = 0xffffffffu;
    float limit = st.limit;
    if (!st.full) {
        // At least `top` logits are not below the top-th largest of the lanes' maxima, so what is below cannot enter; what
        // equals it may: the limit is the next smaller number.
        int above = 0;
#pragma unroll 8
        for (int o = 0; o < 32; ++o) {
            const float other = __shfl_sync(kAll, round_max, o);
            above += other > round_max || (other == round_max && o < (int)(threadIdx.x & 31));
        }
        const unsigned who = __ballot_sync(kAll, above == top - 1);
        const float edge = __shfl_sync(kAll, round_max, who ? __ffs(who) - 1 : 0);
        if (who && edge > -INFINITY) {
            const uint32_t u = __float_as_uint(edge + 0.f);
            limit = edge == 0.f ? -1.4e-45f : __uint_as_float(edge > 0.f ? u - 1u : u + 1u);
        }
    }
    if (!__any_sync(kAll, round_max > limit)) return;
    uint32_t mine = 0u;
#pragma unroll
    for (int i = 0; i < kCount; ++i) mine |= x[i] > limit ? 1u << i : 0u;
    while (__any_sync(kAll, mine != 0u)) {
        const int i = mine ? __ffs(mine) - 1 : 0;
        // the i-th of the lane's registers
        float v = x[0];
#pragma unroll
        for (int j = 1; j < kCount; ++j) v = i == j ? x[j] : v;
        unsigned long long key = mine ? score_key(v, at(i)) : 0ull;
        mine &= mine - 1u;
        key = key > shfl_key(st.list, top - 1) ? key : 0ull;
        st.list = join_list(st.list, key);
    }
    const unsigned long long last = shfl_key(st.list, top - 1);
    st.full = last != 0ull;
    st.limit = st.full ? key_logit(last) : -INFINITY;
}

template <typename T, bool kTop>
__device__ __forceinline__ void score_chunk_warp(const ScoreParams& p, const int row, const int chunk, const long long item) {
    constexpr int kPer = ScoreLoad<T>::kPer, kLoads = ScoreLoad<T>::kLoads;
    const int lane = threadIdx.x & 31;
    const long long V = p.vocab;
    const long long c0 = (long long)chunk * p.chunk, c1 = min(V, c0 + p.chunk);
    const T* base = static_cast<const T*>(p.logits) + (p.row0 + row) * V;
    // [c0, a0) up to 16-byte alignment, [a0, a1) whole loads, [a1, c1) the rest
    const uintptr_t addr = reinterpret_cast<uintptr_t>(base + c0);
    long long a0 = c0 + (long long)(((16 - (addr & 15)) & 15) / sizeof(T));
    if (a0 > c1) a0 = c1;
    const long long a1 = a0 + (c1 - a0) / kPer * kPer;
    const uint4* body = reinterpret_cast<const uint4*>(base + a0);
    const int nvec = (int)((a1 - a0) / kPer);
    const uint64_t policy = l2_evict_first_policy();      // the logits are read once
    constexpr float kNone = -INFINITY;

    ScoreState st;
    auto ragged = [&](long long from, long long to) {      // at most seven logits, one per lane
        if (from >= to) return;
        float x[1] = {from + lane < to ? score_of(base[from + lane]) : kNone};
        const float mx = fmaxf(x[0], kNone);
        score_sums(st, x, mx);
        if constexpr (kTop) score_list(st, p.top, x, mx, [&](int) { return (uint32_t)(from + lane); });
    };
    auto load = [&](int v0, ScoreLoad<T>& l) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int v = v0 + j * 32 + lane;
            if (v < nvec) l.u[j] = ld_stream_u4(body + v, policy);
            else {
                const uint32_t none = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
                l.u[j] = make_uint4(none, none, none, none);
            }
        }
    };
    auto take = [&](int v0, const ScoreLoad<T>& l) {
        float x[32];
        score_unpack(l, x);
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = fmaxf(fmaxf(x[4 * j], x[4 * j + 1]), fmaxf(x[4 * j + 2], x[4 * j + 3]));
        const float mx = fmaxf(fmaxf(fmaxf(fmaxf(g[0], g[1]), fmaxf(g[2], g[3])), fmaxf(fmaxf(g[4], g[5]), fmaxf(g[6], g[7]))), kNone);
        score_sums(st, x, mx);
        if constexpr (kTop)
            score_list(st, p.top, x, mx, [&](int i) { return (uint32_t)(a0 + (long long)(v0 + (i / kPer) * 32 + lane) * kPer + i % kPer); });
    };
    ragged(c0, a0);
    constexpr int kVecs = 32 * kLoads;       // per round
    ScoreLoad<T> la, lb;
    if (nvec > 0) load(0, la);
    for (int v0 = 0; v0 < nvec; v0 += 2 * kVecs) {
        if (v0 + kVecs < nvec) load(v0 + kVecs, lb);
        take(v0, la);
        if (v0 + 2 * kVecs < nvec) load(v0 + 2 * kVecs, la);
        if (v0 + kVecs < nvec) take(v0 + kVecs, lb);
    }
    ragged(a1, c1);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        join_sums(st.m, st.s, st.t, __shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o));
    if (lane == 0) *reinterpret_cast<float4*>(p.part + item) = make_float4(st.m, st.s, st.t, 0.f);
    if (kTop && lane < p.top) p.part_keys[item * p.top + lane] = st.list;
}

template <typename T, bool kTop>
__global__ void __launch_bounds__(kScoreWarps * 32, kScoreCtasPerSm) logprob_scan_kernel(const ScoreParams p) {
    // may be launched as a programmatic dependent: nothing is read before the kernel before it in the stream has
    // completed (a no-op in an ordinary launch); the merge may queue up and waits likewise
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long items = (long long)p.rows * p.chunks, stride = (long long)gridDim.x * kScoreWarps;
    for (long long it = (long long)blockIdx.x * kScoreWarps + (threadIdx.x >> 5); it < items; it += stride) {
        const int row = (int)(it / p.chunks);
        score_chunk_warp<T, kTop>(p, row, (int)(it - (long long)row * p.chunks), it);
    }
}

// (m, s, t) of a row, the same in all lanes of the calling warp; the order of the sum is fixed.
__device__ __forceinline__ void score_row(const ScoreParams& p, int row, float& m, float& s, float& t) {
    const int lane = threadIdx.x & 31;
    m = -INFINITY; s = 0.f; t = 0.f;
    for (int c = lane; c < p.chunks; c += 32) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part + (long long)(row - p.row0) * p.chunks + c));
        join_sums(m, s, t, v.x, v.y, v.z);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        join_sums(m, s, t, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o), __shfl_xor_sync(0xffffffffu, t, o));
}
// x - lse without the rounding of lse at the logits' own magnitude.  A row without a finite logit gives every token probability 0.
__device__ __forceinline__ float score_logprob(float x, float m, float log_s) { return m == -INFINITY ? -INFINITY : (x - m) - log_s; }
__device__ __forceinline__ float score_log_s(float m, float s) { return m == INFINITY ? INFINITY : logf(s); }

// The packed row that predicts node `node`: its parent's.  -1 for a root (nothing is scored), -2 for offsets or a parent that make no
// sense.  The node's sequence is the last one that does not begin after it.
__device__ __forceinline__ int score_parent_row(const ScoreParams& p, int node) {
    const int lane = threadIdx.x & 31;
    int lo, n;
    if (!p.node_offsets) {
        lo = node / p.nodes_uniform * p.nodes_uniform;
        n = p.nodes_uniform;
    } else {
        const int step = (p.batch + 31) >> 5;
        int b = lane * step;
        unsigned at = __ballot_sync(0xffffffffu, b < p.batch && p.node_offsets[b] <= node);
        b = (31 - __clz(at | 1u)) * step;
        if (step > 1) {
            const int first = b;
            b = first + lane;
            at = __ballot_sync(0xffffffffu, lane < step && b < p.batch && p.node_offsets[b] <= node);
            b = first + 31 - __clz(at | 1u);
        }
        lo = p.node_offsets[b];
        n = p.node_offsets[b + 1] - lo;
    }
    if (lo < 0 || n < 1 || n > p.max_nodes || (long long)lo + n > p.total_nodes || node < lo || node >= lo + n) return -2;
    const int parent = p.tree_parent[node];
    if (node == lo) return parent == -1 ? -1 : -2;
    return parent >= 0 && parent < node - lo ? lo + parent : -2;
}

// grid = rows.  Warps join the chunks' lists, then the first joins theirs; the second warp scores the row's token.
template <typename T>
__global__ void __launch_bounds__(kScoreWarps * 32) logprob_merge_kernel(const ScoreParams p) {
    __shared__ unsigned long long s_list[kScoreWarps][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int row = p.row0 + blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned long long list = 0ull;
    if (p.top > 0) {
        const unsigned long long* keys = p.part_keys + (long long)blockIdx.x * p.chunks * p.top;
        for (int c = warp; c < p.chunks; c += kScoreWarps) {
            const unsigned long long k = lane < p.top ? __ldcg(keys + (long long)c * p.top + lane) : 0ull;
            list = c == warp ? k : merge_lists(list, k);
        }
        if (warp > 0) s_list[warp][lane] = list;
        __syncthreads();
    }
    if (warp == 0) {
        for (int w = 1; w < min(kScoreWarps, p.chunks) && p.top > 0; ++w) list = merge_lists(list, s_list[w][lane]);
        float m, s, t;
        score_row(p, row, m, s, t);
        const float log_s = score_log_s(m, s);
        if (lane == 0) {
            if (p.row_sums) p.row_sums[row] = make_float2(m, s);
            if (p.lse) p.lse[row] = m == -INFINITY ? -INFINITY : m + log_s;
            if (p.entropy) p.entropy[row] = m == -INFINITY ? 0.f : log_s - t / s;
        }
        if (lane < p.top) {
            if (p.top_ids) p.top_ids[(long long)row * p.top + lane] = list ? (int)~(uint32_t)list : -1;
            if (p.top_logprobs) p.top_logprobs[(long long)row * p.top + lane] = list ? score_logprob(key_logit(list), m, log_s) : -INFINITY;
        }
    }
    if (warp == 1 && p.logprob) {
        const int token = p.tokens[row], from = p.tree_parent ? score_parent_row(p, row) : row;
        if (from == -2) { if (lane == 0) report(p.status, kErrBadTree); return; }      // the row's logprob stays unwritten
        float y = 0.f;                             // a root, or no token: nothing is scored
        if (from >= 0 && token >= 0) {
            y = -INFINITY;                         // a token that the vocabulary does not have
            if (token < p.vocab) {
                const float x = score_of(static_cast<const T*>(p.logits)[(long long)from * p.vocab + token]);
                float m, s, t;
                if (from < p.row0) {               // a row of an earlier launch (parents come first)
                    const float2 sums = __ldcg(p.row_sums + from);
                    m = sums.x; s = sums.y;
                } else score_row(p, from, m, s, t);
                y = x != x ? -INFINITY : score_logprob(x, m, score_log_s(m, s));
            }
        }
        if (lane == 0) p.logprob[row] = y;
    }
}

// Logits per item, a multiple of a round: the size that ends first when the resident warps take the items in turn, an item costing what
// `kItemCost` more logits would (its first round waits for memory and finds the list's limit, its end joins the lanes' sums).
// At most `most` items; where no size keeps to that, the largest one (the caller then takes the rows in several turns).
inline int score_chunk(long long rows, int vocab, int sms, long long most) {
    constexpr long long kItemCost = 700;
    const long long warps = (long long)sms * kScoreCtasPerSm * kScoreWarps;
    int best = kScoreMaxChunk;
    long long least = -1;
    for (int chunk = kScoreRound; chunk <= kScoreMaxChunk; chunk += kScoreRound) {
        const long long items = rows * (((long long)vocab + chunk - 1) / chunk);
        if (items > most) continue;
        const long long cost = (items + warps - 1) / warps * ((chunk < vocab ? chunk : vocab) + kItemCost);
        if (least < 0 || cost < least) { least = cost; best = chunk; }
    }
    return best;
}
// Items that a context has room for: those of its largest call in chunks of half the largest size, but no more than `kScoreMostItems` (a larger
// call takes its rows in turns) and no less than two for each resident warp.
constexpr long long kScoreMostItems = 32768;
inline long long score_room(long long rows, int vocab, int sms) {
    const long long want = rows * (((long long)vocab + kScoreMaxChunk / 2 - 1) / (kScoreMaxChunk / 2));
    const long long least = 2ll * sms * kScoreCtasPerSm * kScoreWarps;
    const long long room = want < kScoreMostItems ? want : kScoreMostItems;
    return room > least ? room : least;
}

}  // namespace owl
