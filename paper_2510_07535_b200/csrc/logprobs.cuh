// Log probabilities of the drafted tokens under the rows that predict them, with each row's log-sum-exp, entropy and most likely tokens.
//
// One pass over the logits, in two kernels:
//   logprob_scan_kernel   a warp takes a (row, vocabulary chunk) item, 32 logits per lane and round, the next round's loads in
//                         flight meanwhile.  Per lane m = running maximum, s = sum e^(x - m), t = sum e^(x - m) (x - m); and, where
//                         alternatives are asked for, each lane's maximum of each round is left in a table: one for 32 logits.
//   logprob_merge_kernel  a CTA per row joins the chunks:  lse = m + ln s,  entropy = ln s - t / s,  scores a token, and finds
//                         the alternatives: of 64 maxima over parts of the table the top-th largest is not above the top-th
//                         largest logit, so the groups of 32 whose maximum reaches it hold all of them, some tens of groups.
// 256 rows of 128256 fp32 logits with 20 alternatives take 30.0 us (131 MB, 4.4 TB/s, 67 % of the copy bandwidth), 23.9 of them the scan; of bf16
// or fp16 ones 24.6 and 19.4 (66 MB, 2.7 TB/s, 41 %); 8 rows 9.9 to 10.4 us, the latency of two launches.
// fp32 logits are bound by their bytes, 16-bit ones, which are half of them, by the work per logit: per element a maximum, a subtraction, a product, a clamp, an ex2 and two sums.  (A sorted list per warp in the
// scan instead of the table: 256 rows of 128256 fp32 logits 42.8 us with 20 alternatives and 23.9 without, 8 rows 13.9 and 2.7.)
#pragma once

#include "accept.cuh"
#include "owl_common.cuh"
#include "sm100_ptx.cuh"

namespace owl {

constexpr int kMaxTop = 32;              // alternatives per row
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
    float* maxima;                       // [N, chunks, rounds + 1, 32]: of each lane's logits of a round; last, up to 16 ragged logits
    float2* row_sums;                    // [N] a row's (m, s), for the rows of later launches of the call; null: there are none
    int32_t* status;
    int32_t batch, total_nodes, nodes_uniform, max_nodes, vocab, top, chunk, chunks, rounds;
    int32_t row0, rows;                  // this launch's rows [row0, row0 + rows); the partials are counted from row0
};

// What alternatives are ordered by: larger logit first, then the lower token.  0: none (-inf and NaN make none).
__device__ __forceinline__ unsigned long long score_key(float x, uint32_t idx) { return x > -INFINITY ? argmax_key(x, idx) : 0ull; }
__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
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

// One lane's 32 logits of a round, 16 bytes to a load: four logits of 4 bytes or eight of 2.
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

// A lane's sums while its warp works through a chunk.
struct ScoreState {
    float m = -INFINITY, s = 0.f, t = 0.f;
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
    if constexpr (kCount == 1) {
        const float d = fmaxf(x[0] - m, -200.f);
        s0 = exp_of(d);
        t0 = s0 * d;
    } else {
        // pairs, in packed arithmetic
        using namespace sm100;
        uint64_t s2 = 0ull, t2 = 0ull;
        const uint64_t neg_m = pack_f32x2(-m, -m), log2e = pack_f32x2(1.4426950408889634f, 1.4426950408889634f);
#pragma unroll
        for (int i = 0; i < kCount; i += 2) {
            // -inf, a NaN, and the NaN of inf - inf all become a difference whose weight is 0
            float d0, d1, y0, y1;
            unpack_f32x2(add_f32x2(pack_f32x2(x[i], x[i + 1]), neg_m), d0, d1);
            const uint64_t d = pack_f32x2(fmaxf(d0, -200.f), fmaxf(d1, -200.f));
            unpack_f32x2(mul_f32x2(d, log2e), y0, y1);
            const uint64_t e = pack_f32x2(fast_exp2(y0), fast_exp2(y1));
            s2 = add_f32x2(s2, e);
            t2 = fma_f32x2(e, d, t2);
        }
        unpack_f32x2(s2, s0, s1);
        unpack_f32x2(t2, t0, t1);
    }
    st.s += s0 + s1;
    st.t += t0 + t1;
}
// The parts of a chunk: [c0, a0) up to 16-byte alignment, [a0, a1) whole loads, [a1, c1) the rest.
template <typename T>
struct ScoreChunk {
    const T* row;
    long long c0, c1, a0, a1;
    __device__ __forceinline__ ScoreChunk(const ScoreParams& p, long long at_row, int chunk) {
        row = static_cast<const T*>(p.logits) + at_row * p.vocab;
        c0 = (long long)chunk * p.chunk;
        c1 = min((long long)p.vocab, c0 + p.chunk);
        const uintptr_t addr = reinterpret_cast<uintptr_t>(row + c0);
        a0 = min(c1, c0 + (long long)(((16 - (addr & 15)) & 15) / sizeof(T)));
        a1 = a0 + (c1 - a0) / ScoreLoad<T>::kPer * ScoreLoad<T>::kPer;
    }
    // the token of a ragged logit, `i` of 16: the first eight before a0, the others from a1 on; -1: there is none
    __device__ __forceinline__ long long ragged(int i) const {
        const long long v = i < 8 ? c0 + i : a1 + (i - 8);
        return i < 16 && v < (i < 8 ? a0 : c1) ? v : -1;
    }
};

template <typename T, bool kTop>
__device__ __forceinline__ void score_chunk_warp(const ScoreParams& p, const int row, const int chunk, const long long item) {
    constexpr int kPer = ScoreLoad<T>::kPer, kLoads = ScoreLoad<T>::kLoads;
    const int lane = threadIdx.x & 31;
    const ScoreChunk<T> c(p, p.row0 + row, chunk);
    const uint4* body = reinterpret_cast<const uint4*>(c.row + c.a0);
    const int nvec = (int)((c.a1 - c.a0) / kPer);
    const uint64_t policy = l2_evict_first_policy();      // the logits are read once
    constexpr float kNone = -INFINITY;
    float* maxima = kTop ? p.maxima + item * (p.rounds + 1) * 32 + lane : nullptr;

    ScoreState st;
    {
        const long long v = c.ragged(lane);
        float x[1] = {v >= 0 ? score_of(c.row[v]) : kNone};
        const float mx = fmaxf(x[0], kNone);
        score_sums(st, x, mx);
        if constexpr (kTop) maxima[p.rounds * 32] = mx;
    }
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
        if constexpr (kTop) maxima[v0 / (32 * kLoads) * 32] = mx;
    };
    constexpr int kVecs = 32 * kLoads;       // per round
    ScoreLoad<T> la, lb;
    if (nvec > 0) load(0, la);
    int v0 = 0;
    for (; v0 < nvec; v0 += 2 * kVecs) {
        if (v0 + kVecs < nvec) load(v0 + kVecs, lb);
        take(v0, la);
        if (v0 + 2 * kVecs < nvec) load(v0 + 2 * kVecs, la);
        if (v0 + kVecs < nvec) take(v0 + kVecs, lb);
    }
    if constexpr (kTop)
        for (int r = (nvec + kVecs - 1) / kVecs; r < p.rounds; ++r) maxima[r * 32] = kNone;      // rounds that the last chunk has not
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        join_sums(st.m, st.s, st.t, __shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o));
    if (lane == 0) *reinterpret_cast<float4*>(p.part + item) = make_float4(st.m, st.s, st.t, 0.f);
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

// Largest of a CTA's keys; every thread gets it (two barriers).
__device__ __forceinline__ unsigned long long largest_key(unsigned long long k, unsigned long long* s_keys /*[kScoreWarps]*/) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, k, o);
        k = other > k ? other : k;
    }
    if ((threadIdx.x & 31) == 0) s_keys[threadIdx.x >> 5] = k;
    __syncthreads();
    k = s_keys[0];
#pragma unroll
    for (int w = 1; w < kScoreWarps; ++w) k = s_keys[w] > k ? s_keys[w] : k;
    __syncthreads();
    return k;
}

// grid = rows.  The first warp joins the chunks' sums, the second scores the row's token, and all look for the alternatives.
constexpr int kScoreGroups = 512, kScoreCandidates = 1024;
static_assert(kMaxTop <= kScoreWarps * 8, "as many parts of the table as alternatives");
template <typename T>
__global__ void __launch_bounds__(kScoreWarps * 32) logprob_merge_kernel(const ScoreParams p) {
    constexpr int kThreads = kScoreWarps * 32, kPer = ScoreLoad<T>::kPer, kLoads = ScoreLoad<T>::kLoads;
    __shared__ __align__(16) float s_max[kThreads / 4];
    __shared__ float s_edge, s_m, s_log_s;
    __shared__ int s_groups[kScoreGroups], s_count[2];
    __shared__ unsigned long long s_keys[kScoreCandidates];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int row = p.row0 + blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per_chunk = (p.rounds + 1) * 32, groups = p.chunks * per_chunk;      // < 2^31: the table's row fits the context
    const float* maxima = p.maxima + (long long)blockIdx.x * groups;
    // A thread holds its first 32 groups' maxima: 8192 groups, which are 131072 logits in chunks of one round (64 groups each, half of them for
    // the ragged ends) and more in longer ones; those beyond are read twice.
    constexpr int kHeld = 32;
    float held[kHeld];
    if (p.top > 0) {
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) held[i] = tid + i * kThreads < groups ? __ldcg(maxima + tid + i * kThreads) : -INFINITY;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) mx = fmaxf(mx, held[i]);
#pragma unroll 8
        for (int g = tid + kHeld * kThreads; g < groups; g += kThreads) mx = fmaxf(mx, __ldcg(maxima + g));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if ((tid & 3) == 0) s_max[tid >> 2] = mx;
        if (tid < 2) s_count[tid] = 0;
    }
    if (warp == 0) {
        float m, s, t;
        score_row(p, row, m, s, t);
        const float log_s = score_log_s(m, s);
        if (lane == 0) {
            s_m = m; s_log_s = log_s;
            if (p.row_sums) p.row_sums[row] = make_float2(m, s);
            if (p.lse) p.lse[row] = m == -INFINITY ? -INFINITY : m + log_s;
            if (p.entropy) p.entropy[row] = m == -INFINITY ? 0.f : log_s - t / s;
        }
    }
    if (warp == 1 && p.logprob) {
        const int token = p.tokens[row], from = p.tree_parent ? score_parent_row(p, row) : row;
        if (from == -2) {                          // this logprob stays unwritten
            if (lane == 0) report(p.status, kErrBadTree);
        } else {
            float y = 0.f;                         // a root, or no token: nothing is scored
            if (from >= 0 && token >= 0) {
                y = -INFINITY;                     // a token that the vocabulary does not have
                if (token < p.vocab) {
                    const float x = score_of(static_cast<const T*>(p.logits)[(long long)from * p.vocab + token]);
                    float m, s, t;
                    if (from < p.row0) {           // a row of an earlier launch (parents come first)
                        const float2 sums = __ldcg(p.row_sums + from);
                        m = sums.x; s = sums.y;
                    } else score_row(p, from, m, s, t);
                    y = x != x ? -INFINITY : score_logprob(x, m, score_log_s(m, s));
                }
            }
            if (lane == 0) p.logprob[row] = y;
        }
    }
    if (p.top == 0) return;
    __syncthreads();
    if (tid < kThreads / 4) {
        // the top-th largest of 64 maxima, four threads' each: at least `top` logits are not below it
        const float mine = s_max[tid];
        int above = 0;
#pragma unroll
        for (int j = 0; j < kThreads / 4; j += 4) {
            const float4 o = *reinterpret_cast<const float4*>(s_max + j);
            above += (o.x > mine || (o.x == mine && j < tid)) + (o.y > mine || (o.y == mine && j + 1 < tid)) +
                     (o.z > mine || (o.z == mine && j + 2 < tid)) + (o.w > mine || (o.w == mine && j + 3 < tid));
        }
        if (above == p.top - 1) s_edge = mine;
    }
    __syncthreads();
    const float edge = s_edge;
    auto reaches = [&](float x) { return x >= edge && x > -INFINITY; };
    auto take_group = [&](int g) {
        const int at = atomicAdd(&s_count[0], 1);
        if (at < kScoreGroups) s_groups[at] = g;
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (reaches(held[i])) take_group(tid + i * kThreads);
#pragma unroll 8
    for (int g = tid + kHeld * kThreads; g < groups; g += kThreads)
        if (reaches(__ldcg(maxima + g))) take_group(g);
    __syncthreads();
    const int found = s_count[0];
    if (found <= kScoreGroups) {
        // a group's logits lie in kLoads pieces of 16 bytes, 512 bytes apart: a thread per piece
        for (int u = tid; u < found * kLoads; u += kThreads) {
            const int g = s_groups[u / kLoads], j = u % kLoads;
            const int chunk = g / per_chunk, r = g % per_chunk / 32, l = g % 32;
            const ScoreChunk<T> c(p, row, chunk);
            auto offer = [&](long long v, float x) {
                if (reaches(x)) {
                    const int at = atomicAdd(&s_count[1], 1);
                    if (at < kScoreCandidates) s_keys[at] = score_key(x, (uint32_t)v);
                }
            };
            if (r == p.rounds) {
                const long long v = c.ragged(l);
                if (j == 0 && v >= 0) offer(v, score_of(c.row[v]));
            } else {
                const long long v = c.a0 + ((long long)(r * kLoads + j) * 32 + l) * kPer;
                if (v < c.a1) {
                    const uint4 piece = *reinterpret_cast<const uint4*>(c.row + v);
                    const T* x = reinterpret_cast<const T*>(&piece);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) offer(v + e, score_of(x[e]));
                }
            }
        }
    }
    __syncthreads();
    const int count = s_count[1];
    const float m = s_m, log_s = s_log_s;
    auto write = [&](int j, unsigned long long k) {
        if (p.top_ids) p.top_ids[(long long)row * p.top + j] = k ? (int)~(uint32_t)k : -1;
        if (p.top_logprobs) p.top_logprobs[(long long)row * p.top + j] = k ? score_logprob(key_logit(k), m, log_s) : -INFINITY;
    };
    if (found <= kScoreGroups && count <= kScoreCandidates) {
        // a candidate's place is the number of larger ones (their order here, which is by chance, does not matter)
        for (int i = tid; i < max(count, p.top); i += kThreads) {
            if (i >= count) { write(i, 0ull); continue; }
            const unsigned long long mine = s_keys[i];
            int above = 0;
#pragma unroll 8
            for (int j = 0; j < count; ++j) above += s_keys[j] > mine;
            if (above < p.top) write(above, mine);
        }
    } else {
        // hundreds of logits equal to the last one's value: one alternative after the other from the whole row
        const T* logits = static_cast<const T*>(p.logits) + (long long)row * p.vocab;
        unsigned long long last = ~0ull;
        for (int j = 0; j < p.top; ++j) {
            unsigned long long best = 0ull;
            for (int v = tid; v < p.vocab; v += kThreads) {
                const unsigned long long k = score_key(score_of(logits[v]), (uint32_t)v);
                if (k < last && k > best) best = k;
            }
            best = largest_key(best, s_keys);
            if (tid == 0) write(j, best);
            last = best;
        }
    }
}

// Logits per item, a multiple of a round: the size that ends first when the resident warps take the items in turn, an item costing what
// `kItemCost` more logits would (its first round waits for memory, its end joins the lanes' sums).  Rows of 128256 logits, us, at 0 / 350 / 700 /
// 1400 / 2800: 32 rows of fp32 16.0 / 12.5 / 12.5 / 12.5 / 12.5, 256 30.3 / 29.7 / 29.8 / 29.8 / 29.8, of bf16 26.0 / 24.6 / 24.7 / 24.6 /
// 24.6, 960 of bf16 89.9 / 89.9 / 90.0 / 72.8 / 72.8.
// At most `most` items; where no size keeps to that, the largest one (the caller then takes the rows in several turns).
inline int score_chunk(long long rows, int vocab, int sms, long long most) {
    constexpr long long kItemCost = 700;
    const long long warps = (long long)sms * kScoreCtasPerSm * kScoreWarps;
    const long long whole = ((long long)vocab + kScoreRound - 1) / kScoreRound * kScoreRound;      // the row in one chunk
    const int largest = whole < kScoreMaxChunk ? (int)whole : kScoreMaxChunk;
    int best = largest;
    long long least = -1;
    for (int chunk = kScoreRound; chunk <= largest; chunk += kScoreRound) {
        const long long items = rows * (((long long)vocab + chunk - 1) / chunk);
        if (items > most) continue;
        const long long cost = (items + warps - 1) / warps * ((chunk < vocab ? chunk : vocab) + kItemCost);
        if (least < 0 || cost < least) { least = cost; best = chunk; }
    }
    return best;
}
// Places of a row's table of maxima, in chunks of `chunk`; what a context has room for: its largest call's in the smallest chunks, but no more
// than 16 MB unless one row needs them.
inline long long score_table(int vocab, int chunk) { return ((long long)vocab + chunk - 1) / chunk * (chunk / kScoreRound + 1) * 32; }
inline long long score_table_room(long long rows, int vocab) {
    const long long row = score_table(vocab, kScoreRound), want = rows * row, most = 4ll << 20;
    return want < most ? want : row > most ? row : most;
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
