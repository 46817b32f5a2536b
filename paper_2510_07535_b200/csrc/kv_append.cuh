// New tokens on their way from the projections to the verify pass: queries and keys are turned by their positions, keys and values
// written to the paged cache at logical positions L .. L + n - 1 (drafts, or a prompt), in the cache's 16-bit type or in 8 bits
// with a power-of-two scale per page and head (fp8_block.cuh).  The inputs are read once, every output is written once.
//
// Rotation: element j of the first half and j of the second half of a head (64 apart) are turned by the angle of the token's
// position, taken from the caller's table of cosines and sines in fp32:
//     x'_j = x_j cos_j - x_{j+64} sin_j,   x'_{j+64} = x_{j+64} cos_j + x_j sin_j
// each product and the sum rounded to fp32 by itself (no contraction, so the bits do not depend on the compiler), then once to
// the output's type.
//
// A CTA has one page of one sequence and some of its heads: thread = (slot of the page, eight elements of each half), so its
// table entries stay in registers over all its heads, and a block's largest magnitude is a reduction over the CTA.  Items
// (pages) are numbered without a prefix sum over the batch: sequence b's begin at floor(offset_b / page) + 2 b, because
// n tokens touch at most floor(n / page) + 2 pages wherever they begin.
//
// Bound by the rows' bytes for a prompt, by one chain of dependent loads (offsets, length, table, row) for a draft: 8191 tokens to 8
// bits with 32 + 16 heads take 38.5 us (189 MB, 4.9 TB/s, 75 % of the copy bandwidth), four prompts of 2047 in fp16 63.6 us (340 MB,
// 5.3 TB/s, 81 %; to 8 bits a barrier stands between a head's loads and its stores, and 16 bytes spill under the 64 registers that
// 1024 threads leave), a chain of 8 or 16 trees of 32 about 3 and 5 us on the device and 9.3 us from call to call, which is the host's.
#pragma once

#include "fp8_block.cuh"
#include "owl_common.cuh"

namespace owl {

struct AppendParams {
    const __nv_bfloat16* q;        // may be null; bf16 or fp16 (typed as bf16 pointers here)
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    long long q_stride, k_stride, v_stride;      // elements from one token's row to the next
    const int32_t* positions;      // may be null: L + index in the sequence
    const float* rope;             // [rope_rows, 128] 64 cosines, 64 sines; null: nothing is turned
    __nv_bfloat16* q_out;          // [N, Hq, 128]
    void* k_cache;
    void* v_cache;
    int8_t* page_exp;              // 8-bit cache: [num_pages, Hkv, 2] exponents of K and V
    const int32_t* block_table;
    const int32_t* ctx_lens;
    const int32_t* node_offsets;   // may be null
    int32_t* status;
    int32_t rope_rows, batch, total_nodes, nodes_uniform, num_q_heads, num_kv_heads;
    int32_t page_size, page_shift, max_pages_per_seq, num_pages;
    int32_t kv_groups, kv_heads_per_group, q_heads_per_group;      // grid.y = kv_groups, then the groups of query heads
};

constexpr int kAppendMaxWarps = 32;      // of a CTA: 8 threads per slot, pages of up to 128

template <bool kF16>
__device__ __forceinline__ void unpack_16bit(uint32_t u, float& x, float& y) {
    if (kF16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
        x = f.x; y = f.y;
    } else {
        x = __uint_as_float(u << 16); y = __uint_as_float(u & 0xffff0000u);
    }
}
template <bool kF16>
__device__ __forceinline__ uint32_t round_16bit(float x, float y) {
    if (kF16) { __half2 h = __floats2half2_rn(x, y); return *reinterpret_cast<uint32_t*>(&h); }
    __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&b);
}
template <bool kF16>
__device__ __forceinline__ void unpack8(const uint4& u, float (&x)[8]) {
    unpack_16bit<kF16>(u.x, x[0], x[1]); unpack_16bit<kF16>(u.y, x[2], x[3]);
    unpack_16bit<kF16>(u.z, x[4], x[5]); unpack_16bit<kF16>(u.w, x[6], x[7]);
}
template <bool kF16>
__device__ __forceinline__ uint4 round8(const float (&x)[8]) {
    return make_uint4(round_16bit<kF16>(x[0], x[1]), round_16bit<kF16>(x[2], x[3]), round_16bit<kF16>(x[4], x[5]), round_16bit<kF16>(x[6], x[7]));
}

// a = the thread's elements of the first half, b = of the second
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        a[i] = __fsub_rn(__fmul_rn(x, cs[i]), __fmul_rn(y, sn[i]));
        b[i] = __fadd_rn(__fmul_rn(y, cs[i]), __fmul_rn(x, sn[i]));
    }
}
// Largest magnitude of 16 values, as bits; a NaN counts for nothing.
__device__ __forceinline__ uint32_t magnitude16(const float (&a)[8], const float (&b)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fmaxf(fabsf(a[i]), fabsf(b[i])));
    return __float_as_uint(m);
}
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inv) {
    return make_uint2(pack_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), pack_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
}

// The sequence that item `item` belongs to (all lanes of a warp get it): the last one whose items do not begin after it.
// 32 sequences are looked at at a time: one round of loads for up to 32, two for up to 1024.
__device__ __forceinline__ int append_offset(const AppendParams& p, int b) {
    return p.node_offsets ? p.node_offsets[b] : b * p.nodes_uniform;
}
__device__ __forceinline__ int append_first_item(const AppendParams& p, int b) { return (append_offset(p, b) >> p.page_shift) + 2 * b; }
__device__ __forceinline__ int append_sequence(const AppendParams& p, int item) {
    const int lane = threadIdx.x & 31;
    const int step = (p.batch + 31) >> 5;
    int b = lane * step;
    unsigned at = __ballot_sync(0xffffffffu, b < p.batch && append_first_item(p, b) <= item);
    const int first = (31 - __clz(at | 1u)) * step;
    if (step == 1) return first;
    b = first + lane;
    at = __ballot_sync(0xffffffffu, lane < step && b < p.batch && append_first_item(p, b) <= item);
    return first + 31 - __clz(at | 1u);
}

// grid (items, groups of KV heads then of query heads), 8 threads per slot of a page
template <bool kF16, bool kFp8>
__global__ void __launch_bounds__(1024) kv_append_kernel(const AppendParams p) {
    // may be launched as a programmatic dependent: nothing is read before the kernel before it in the stream has
    // completed (a no-op in an ordinary launch); the kernel after this one may queue up and waits likewise
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ uint32_t s_most[2][2][kAppendMaxWarps];      // [turn][K, V][warp]
    const int tid = threadIdx.x, slot = tid >> 3, c = tid & 7;
    if (blockIdx.x == 0 && blockIdx.y == 0 && p.node_offsets) {
        // do the packed offsets describe the call's rows?  (What they would put out of range is not touched below.)
        bool bad = false;
        for (int b = tid; b < p.batch; b += blockDim.x) {
            const int lo = p.node_offsets[b], hi = p.node_offsets[b + 1];
            bad = bad || hi < lo || (b == 0 && lo != 0) || (b == p.batch - 1 && hi != p.total_nodes);
        }
        if (bad) report(p.status, kErrBadTree);
    }
    const int b = append_sequence(p, (int)blockIdx.x);
    const int base = append_offset(p, b), n = append_offset(p, b + 1) - base;
    const int L = p.ctx_lens[b];
    const int item = (int)blockIdx.x - append_first_item(p, b);
    if (n < 1 || base < 0 || (long long)base + n > p.total_nodes || item < 0) return;
    if (L < 0 || (long long)L + n > min((long long)p.max_pages_per_seq * p.page_size, 0x7fffff00ll)) {
        if (tid == 0 && item == 0) report(p.status, kErrBadPage);
        return;                                     // the sequence does not fit its row of the table: nothing of it is written
    }
    const int lp = (L >> p.page_shift) + item;
    if (lp > (L + n - 1) >> p.page_shift) return;
    const int page = p.block_table[(long long)b * p.max_pages_per_seq + lp];
    const int pos = (lp << p.page_shift) + slot, i = pos - L;       // (no overflow: L + n <= 2^31 - 256)
    bool fresh = i >= 0 && i < n;                   // this thread's slot gets a new token
    const long long token = base + i;
    float cs[8], sn[8];
    if (p.rope && fresh) {
        const int at = p.positions ? p.positions[token] : pos;
        if ((unsigned)at < (unsigned)p.rope_rows) {
            const float4* row = reinterpret_cast<const float4*>(p.rope + (long long)at * kHeadDim + 8 * c);
            const float4 c0 = __ldg(row), c1 = __ldg(row + 1), s0 = __ldg(row + 16), s1 = __ldg(row + 17);
            cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
            sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
        } else {
            report(p.status, kErrBadPage);          // a position that the table does not have: the token is left out
            fresh = false;
        }
    }
    const bool turned = p.rope != nullptr;

    if ((int)blockIdx.y >= p.kv_groups) {           // query heads
        const int h0 = ((int)blockIdx.y - p.kv_groups) * p.q_heads_per_group, h1 = min(p.num_q_heads, h0 + p.q_heads_per_group);
        if (!fresh) return;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + token * p.q_stride) + c;
        uint4* dst = reinterpret_cast<uint4*>(p.q_out + token * p.num_q_heads * kHeadDim) + c;
#pragma unroll 4
        for (int h = h0; h < h1; ++h) {
            uint4 ua = src[h * 16], ub = src[h * 16 + 8];
            if (turned) {
                float a[8], d[8];
                unpack8<kF16>(ua, a); unpack8<kF16>(ub, d);
                turn(a, d, cs, sn);
                ua = round8<kF16>(a); ub = round8<kF16>(d);
            }
            dst[h * 16] = ua;
            dst[h * 16 + 8] = ub;
        }
        return;
    }

    if ((unsigned)page >= (unsigned)p.num_pages) {  // the same for the whole CTA: the page's tokens are left out
        if (tid == 0) report(p.status, kErrBadPage);
        return;
    }
    const int h0 = (int)blockIdx.y * p.kv_heads_per_group, h1 = min(p.num_kv_heads, h0 + p.kv_heads_per_group);
    const uint4* ksrc = reinterpret_cast<const uint4*>(p.k + token * p.k_stride) + c;
    const uint4* vsrc = reinterpret_cast<const uint4*>(p.v + token * p.v_stride) + c;
    if constexpr (!kFp8) {
        if (!fresh) return;
#pragma unroll 2
        for (int h = h0; h < h1; ++h) {
            uint4 ka = ksrc[h * 16], kb = ksrc[h * 16 + 8];
            const uint4 va = vsrc[h * 16], vb = vsrc[h * 16 + 8];
            if (turned) {
                float a[8], d[8];
                unpack8<kF16>(ka, a); unpack8<kF16>(kb, d);
                turn(a, d, cs, sn);
                ka = round8<kF16>(a); kb = round8<kF16>(d);
            }
            const long long row = (((long long)page * p.num_kv_heads + h) * p.page_size + slot) * 16 + c;      // in 16-byte pieces
            uint4* kd = static_cast<uint4*>(p.k_cache) + row;
            uint4* vd = static_cast<uint4*>(p.v_cache) + row;
            kd[0] = ka; kd[8] = kb;
            vd[0] = va; vd[8] = vb;
        }
    } else {
        const bool old = pos < L;                   // a row of the context on the page that the new tokens begin on
        const bool begins = (lp << p.page_shift) >= L;      // the page holds nothing yet: what its exponents were says nothing
        const int warps = blockDim.x >> 5;
        for (int h = h0; h < h1; ++h) {
            const long long block = (long long)page * p.num_kv_heads + h;
            const int8_t* exps = p.page_exp + block * 2;
            const int had[2] = {begins ? kExpMin : read_exponent(exps), begins ? kExpMin : read_exponent(exps + 1)};
            float x[2][2][8];                       // [K, V][half]
            uint32_t most[2] = {0u, 0u};
            if (fresh) {
                unpack8<kF16>(ksrc[h * 16], x[0][0]); unpack8<kF16>(ksrc[h * 16 + 8], x[0][1]);
                unpack8<kF16>(vsrc[h * 16], x[1][0]); unpack8<kF16>(vsrc[h * 16 + 8], x[1][1]);
                if (turned) turn(x[0][0], x[0][1], cs, sn);
                most[0] = magnitude16(x[0][0], x[0][1]);
                most[1] = magnitude16(x[1][0], x[1][1]);
            }
            // (two sets of places in turn: a warp that is ahead writes the next head's while another still reads these)
            const int set = (h - h0) & 1;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                most[kv] = __reduce_max_sync(0xffffffffu, most[kv]);      // non-negative floats compare as their bits
                if ((tid & 31) == 0) s_most[set][kv][tid >> 5] = most[kv];
            }
            __syncthreads();
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                uint32_t m = 0u;
                for (int w = 0; w < warps; ++w) m = max(m, s_most[set][kv][w]);
                const int need = block_exponent(m), e = max(had[kv], need);
                uint2* row = reinterpret_cast<uint2*>(static_cast<uint8_t*>(kv ? p.v_cache : p.k_cache) + (block * p.page_size + slot) * kHeadDim) + c;
                if (fresh) {
                    const float inv = exp2_int(-e);
                    row[0] = encode8(x[kv][0], inv);
                    row[8] = encode8(x[kv][1], inv);
                } else if (old && e > had[kv]) {
                    const float f = exp2_int(had[kv] - e);
                    const uint2 a = row[0], d = row[8];
                    row[0] = make_uint2(rescale_e4m3x4(a.x, f), rescale_e4m3x4(a.y, f));
                    row[8] = make_uint2(rescale_e4m3x4(d.x, f), rescale_e4m3x4(d.y, f));
                }
                if (tid == 0) p.page_exp[block * 2 + kv] = (int8_t)e;
            }
        }
    }
}

// Heads per CTA: as few as still give the device a quarter of the CTAs that it holds at once (a draft: one, its latency counts), more where the
// pages alone are enough: what a CTA finds out before it can ask for its first row - sequence, page, position, table entry - is
// four loads one after the other.  (Four prompts of 2047 in fp16, all CTAs that are resident / a quarter: 67.0 / 64.0 us;
// one of 8191 to 8 bits 38.4 / 38.9.)
inline int append_heads_per_group(long long items, int heads, int page_size, int sms) {
    const long long want = (long long)sms * (2048 / (8 * page_size)) / 4;
    long long groups = (want + items - 1) / items;
    if (groups > heads) groups = heads;
    if (groups < 1) groups = 1;
    return (int)((heads + groups - 1) / groups);
}

}  // namespace owl
