// The commit of accepted tokens (spec_loop.cuh) in the 8-bit cache: a row that moves may come onto a page of another exponent.
// The page takes the larger of its exponent and what the rows that move there need; where that is a larger one, the rows that
// stay on the page - the context's and the accepted ones that lie right already - are re-encoded.  Rows that are neither
// (drafts left behind) keep their bytes.
#pragma once

#include "fp8_block.cuh"
#include "spec_loop.cuh"

namespace owl {

struct CommitFp8Params {
    CommitParams base;             // the caches as pointers to bytes
    int8_t* page_exp;              // [num_pages, Hkv, 2]
};

// Largest magnitude of 16 e4m3, as a byte without sign; a NaN (0x7f) counts for nothing.
__device__ __forceinline__ uint32_t magnitude_e4m3x16(const uint4& u) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = (i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w) & 0x7f7f7f7fu;
        m = __vmaxu4(m, w & ~__vcmpeq4(w, 0x7f7f7f7fu));
    }
    m = max(m & 0xffu, max((m >> 8) & 0xffu, max((m >> 16) & 0xffu, m >> 24)));
    return m;
}
__device__ __forceinline__ uint4 rescale_e4m3x16(const uint4& u, float f) {
    return make_uint4(rescale_e4m3x4(u.x, f), rescale_e4m3x4(u.y, f), rescale_e4m3x4(u.z, f), rescale_e4m3x4(u.w, f));
}

// Bound by latency, the exponents (a load behind the table's) and the rows: 3.4 us for one tree of 32, 4.5 for 64 trees, 9.5 us from
// call to call.
// grid and clusters as kv_commit_kernel: a sequence's heads are dealt out to its cluster's CTAs, half of a CTA's threads move K,
// half V, eight threads (16 bytes each) to a row.
__global__ void __launch_bounds__(kCommitThreads) kv_commit_fp8_kernel(const CommitFp8Params fp) {
    // may be launched as a programmatic dependent: nothing is read before the kernel before it in the stream has
    // completed (a no-op in an ordinary launch); the kernel after this one may queue up and waits likewise
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const CommitParams& p = fp.base;
    __shared__ uint4 s_rows[2][kMaxNodes * 8];
    __shared__ int s_path[kMaxNodes];
    __shared__ int s_pages[kCommitPages];
    __shared__ int s_had[2][kCommitPages], s_exp[2][kCommitPages];
    const int b = blockIdx.y;
    int L, n, a;
    const int verdict = commit_verdict(p, b, L, n, a, s_path, s_pages);
    if (verdict != 0) {                            // in every CTA of the cluster
        if (threadIdx.x == 0 && blockIdx.x == 0) report(p.status, verdict);
        return;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // this CTA has read the length
    constexpr int kHalf = kCommitThreads / 2;
    const int kv = threadIdx.x / kHalf, t = threadIdx.x % kHalf, first = t >> 3, piece = t & 7;
    constexpr int kStep = kHalf / 8;               // rows per turn of a half
    uint8_t* cache = reinterpret_cast<uint8_t*>(kv ? p.v_cache : p.k_cache);
    const int first_page = L >> p.page_shift, pages = ((L + n - 1) >> p.page_shift) - first_page + 1;
    // the path ascends from node 0: its first `stays` nodes lie where they belong, all later ones come from further on
    const int stays = __syncthreads_count(threadIdx.x < a && s_path[threadIdx.x] == (int)threadIdx.x);
    for (int h = blockIdx.x; stays < a && h < p.num_kv_heads; h += gridDim.x) {
        auto row_ptr = [&](int pos) {
            const long long page = s_pages[(pos >> p.page_shift) - first_page];
            return reinterpret_cast<uint4*>(cache + ((page * p.num_kv_heads + h) * p.page_size + (pos & (p.page_size - 1))) * kHeadDim) + piece;
        };
        if (t < pages) s_had[kv][t] = s_exp[kv][t] = read_exponent(fp.page_exp + ((long long)s_pages[t] * p.num_kv_heads + h) * 2 + kv);
        __syncthreads();
        // every row that moves is read before any is written: a position can be the source of one move and the destination of
        // another
        for (int k = stays + first; k < a; k += kStep) {
            const int from = L + s_path[k];
            const uint4 row = *row_ptr(from);
            s_rows[kv][k * 8 + piece] = row;
            uint32_t m = magnitude_e4m3x16(row);
            const unsigned peers = 0xffu << (threadIdx.x & 24);      // the row's eight threads (they take the same turns)
            m = __reduce_max_sync(peers, m);
            if (piece == 0) {
                const float most = e4m3x4_to_f32(m).x * exp2_int(s_had[kv][(from >> p.page_shift) - first_page]);
                atomicMax(&s_exp[kv][((L + k) >> p.page_shift) - first_page], block_exponent(__float_as_uint(most)));
            }
        }
        __syncthreads();
        for (int g = 0; g < pages; ++g) {
            const int had = s_had[kv][g], e = s_exp[kv][g];
            if (e == had) continue;
            const int at = (first_page + g) << p.page_shift, end = min(at + p.page_size, L + stays);
            for (int pos = at + first; pos < end; pos += kStep) *row_ptr(pos) = rescale_e4m3x16(*row_ptr(pos), exp2_int(had - e));
        }
        for (int k = stays + first; k < a; k += kStep) {      // (a thread takes back what it put there itself)
            const int from = s_had[kv][((L + s_path[k]) >> p.page_shift) - first_page], to = s_exp[kv][((L + k) >> p.page_shift) - first_page];
            uint4 row = s_rows[kv][k * 8 + piece];
            if (from != to) row = rescale_e4m3x16(row, exp2_int(from - to));
            *row_ptr(L + k) = row;
        }
        if (t < pages && s_exp[kv][t] != s_had[kv][t])
            fp.page_exp[((long long)s_pages[t] * p.num_kv_heads + h) * 2 + kv] = (int8_t)s_exp[kv][t];
        __syncthreads();                           // the next head's exponents take these places
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) p.ctx_lens[b] = L + a;
}

}  // namespace owl
