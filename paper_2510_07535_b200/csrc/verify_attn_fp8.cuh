// Verify attention over the 8-bit cache (fp8_block.cuh): the pass of verify_attn_umma.cuh - its partition, segments, products, softmax
// and partials - with four more warps between the copies and the products.
//
//   warp 0        TMA producer: one box per (page, head) of K and of V into a ring of 16 KB raw slots; leaves each tile's exponents
//   warp 1        issues the products (mma_loop)
//   warps 4-11    softmax (softmax_loop)
//   warps 12-15   turn a raw slot into an fp16 operand tile: e4m3 * 2^e is an fp16 number, so nothing is rounded (but what lies
//                 below fp16's smallest step, 2^-24), and both products are the 16-bit ones of the 16-bit caches, exact in their operands.
//                 (Products of 8-bit operands straight from the raw slots would need queries and weights cut into e4m3
//                 pieces: twice the instructions at twice the rate, and weights below 2^-15 of the largest would be lost, which
//                 is where a long context's mass may lie beside one dominant key.)
//
// HBM brings half the bytes of a 16-bit cache; what a tile costs the SM in shared-memory traffic is more than there: 32 KB written by TMA,
// 32 read and 64 written by the conversion, then Q, K and V as operands.
#pragma once

#include "fp8_block.cuh"
#include "verify_attn_umma.cuh"

namespace owl {
namespace umma_path {

constexpr int kFp8Threads = 512;
constexpr int kRawBytes = kTileKeys * kHeadDim;      // 16 KB
template <bool kWide> constexpr int kRawSlots = kWide ? 2 : kFp8RawSlots;
template <bool kWide> constexpr int kRawOff = kRingOff<kWide> + kFp8Slots * kSlotBytes;
static_assert(kRawOff<false> + kRawSlots<false> * kRawBytes == kAuxOff && kRawOff<true> + kRawSlots<true> * kRawBytes == kAuxOff, "layout");

template <bool kWide, bool kManySeqs>
__device__ __forceinline__ void producer_loop_fp8(const AttnParams& p, const CUtensorMap* kmap, const CUtensorMap* vmap, AuxFp8* aux,
                                                  uint32_t raw, Walker<kManySeqs> w) {
    constexpr uint32_t kPlaces = kRawSlots<kWide> / 2;
    const int lane = threadIdx.x & 31;
    volatile int* abort_flag = &aux->abort_flag;
    const int ppt = kTileKeys >> p.page_shift;               // pages (= TMA boxes) per tile
    const uint32_t box_bytes = (uint32_t)p.page_size * 128u;
    const int oob = p.num_pages * p.num_kv_heads;            // a coordinate past the end: the box reads zeros
    const uint64_t stream_policy = l2_policy_evict_first();
    uint32_t place = 0, free_parity = 1;
    for (uint32_t seg_no = 0;; ++seg_no) {
        Segment g;
        g.b = g.n = g.L = 0;
        const bool more = w.template next<kWide>(p, g);
        const int keys = g.L + g.n;
        const int pages_valid = (keys + p.page_size - 1) >> p.page_shift;
        const int32_t* table = p.block_table + (long long)g.b * p.max_pages_per_seq;
        auto page_of = [&](int t) {
            const int lp = t * ppt + lane;
            return lane < ppt && lp < pages_valid ? table[lp] : -1;
        };
        // K's exponent in the low byte, V's in the high one
        auto exps_of = [&](int pg) -> int {
            return (unsigned)pg < (unsigned)p.num_pages ? *reinterpret_cast<const uint16_t*>(p.page_exp + ((long long)pg * p.num_kv_heads + g.h) * 2) : 0;
        };
        // pages are asked for two tiles ahead and their exponents one tile ahead
        int page_cur = more ? page_of(g.tile0) : -1, page_next = more && g.tile0 + 1 < g.tile1 ? page_of(g.tile0 + 1) : -1;
        if (seg_no >= (uint32_t)kSegs && !readers_reached(aux, (int)seg_no - kSegs + 1)) break;
        Segment& announced = aux->seg[seg_no % kSegs];
        if (lane == 0) {
            if (!more) g.tile0 = g.tile1 = 0;
            g.bad_page = 0;
            announced = g;
            mbar_arrive(smem_u32(&aux->seg_full[seg_no % kSegs]));
        }
        __syncwarp();
        if (!more) break;
        int exps_cur = exps_of(page_cur);
        for (int t = g.tile0; t < g.tile1; ++t) {
            int coord = oob;
            if ((unsigned)page_cur < (unsigned)p.num_pages) coord = page_cur * p.num_kv_heads + g.h;
            else if (lane < ppt && t * ppt + lane < pages_valid) {
                report(p.status, kErrBadPage);
                const_cast<volatile int&>(announced.bad_page) = 1;
            }
            const int exps_next = exps_of(page_next);
            const int page_after = t + 2 < g.tile1 ? page_of(t + 2) : -1;
            bool ok = true;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const uint32_t slot = 2u * place + kv, full = smem_u32(&aux->raw_full[slot]);
                ok = mbar_wait(smem_u32(&aux->raw_empty[slot]), free_parity, abort_flag) && ok;
                if (ok && lane == 0) mbar_arrive_expect_tx(full, (uint32_t)kRawBytes);
                __syncwarp();
                if (ok && lane < ppt)
                    tma_load_3d_hint(raw + slot * kRawBytes + lane * box_bytes, kv ? vmap : kmap, full, 0, 0, coord, stream_policy);
                __syncwarp();
            }
            // V's slot is free, so the warps that read this place's note are done with it; the K slot's barrier expects one more arrival
            TileNote& note = aux->note[place];
            if (lane < ppt) {
                note.exp[0][lane] = (int8_t)(exps_cur & 0xff);
                note.exp[1][lane] = (int8_t)(exps_cur >> 8);
            }
            if (lane == 0) note.valid = min(kTileKeys, keys - t * kTileKeys);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&aux->raw_full[2u * place]));
            page_cur = page_next; page_next = page_after; exps_cur = exps_next;
            if (++place == kPlaces) { place = 0; free_parity ^= 1u; }
        }
    }
    // no more tiles (after a wait that gave up the converting warps stop by themselves)
    const bool ok = mbar_wait(smem_u32(&aux->raw_empty[2u * place]), free_parity, abort_flag) &&
                    mbar_wait(smem_u32(&aux->raw_empty[2u * place + 1u]), free_parity, abort_flag);
    if (lane == 0 && ok) {
        aux->note[place].valid = -1;
        mbar_arrive(smem_u32(&aux->raw_full[2u * place]));
        mbar_arrive(smem_u32(&aux->raw_full[2u * place]));
    }
}

// ------------------------------------------------------------------------------------------ conversion
// Warp w of four takes key groups 4w .. 4w + 3 of a tile, eight keys x 64 elements per turn.  Lane: 16 elements (one 16-byte piece) of
// one key.  Raw rows are 128 bytes with piece x at place x ^ (key & 7), operand rows 128 bytes per half of the head dimension with
// piece y at y ^ (key & 7), and a raw piece becomes operand pieces 2x, 2x + 1: eight neighbouring lanes take four pieces of two keys
// that differ in bits 0 and 2, so that neither the loads nor the stores meet in a bank.
template <bool kWide>
__device__ __forceinline__ void convert_loop(const AttnParams& p, AuxFp8* aux, unsigned char* smem) {
    constexpr uint32_t kPlaces = kRawSlots<kWide> / 2;
    constexpr unsigned kAll = 0xffffffffu;
    volatile int* abort_flag = &aux->abort_flag;
    const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
    const int r = lane >> 2, key7 = (r >> 1) ^ ((r & 1) * 5), piece = lane & 3;
    const unsigned char* raw = smem + kRawOff<kWide> + warp * 4096 + key7 * 128;
    unsigned char* ring = smem + kRingOff<kWide> + warp * 8192 + key7 * 128;
    for (uint32_t n = 0;; ++n) {
        const uint32_t place = n % kPlaces, parity = (n / kPlaces) & 1u;
        if (!__all_sync(kAll, mbar_wait(smem_u32(&aux->raw_full[2u * place]), parity, abort_flag))) return;
        const TileNote& note = aux->note[place];
        const int valid = const_cast<const volatile int&>(note.valid);
        if (valid < 0) return;
#pragma unroll 1
        for (uint32_t kv = 0; kv < 2; ++kv) {
            const uint32_t slot = 2u * (n % kFp8Places) + kv;
            bool ok = kv == 0 || mbar_wait(smem_u32(&aux->raw_full[2u * place + 1u]), parity, abort_flag);
            ok = mbar_wait(smem_u32(&aux->empty[slot]), ((n / kFp8Places) & 1u) ^ 1u, abort_flag) && ok;
            if (!__all_sync(kAll, ok)) return;
            const unsigned char* src = raw + (2u * place + kv) * kRawBytes;
            unsigned char* dst = ring + slot * kSlotBytes;
            uint4 u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                u[j] = *reinterpret_cast<const uint4*>(src + (j >> 1) * 1024 + ((((j & 1) * 4 + piece) ^ key7) << 4));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = (4 * warp + (j >> 1)) * 8;             // of the group's first key
                const int e = max(kExpMin, min(kExpMax, (int)note.exp[kv][key >> p.page_shift]));
                const uint32_t one = e >= -14 ? (uint32_t)(e + 15) << 10 : 1u << (e + 24);
                const uint32_t two_to_e = one | one << 16;
                uint32_t o[8];
                const uint32_t w[4] = {u[j].x, u[j].y, u[j].z, u[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a = e4m3x2_to_f16x2(w[i] & 0xffffu), b = e4m3x2_to_f16x2(w[i] >> 16);
                    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * i]) : "r"(a), "r"(two_to_e));
                    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * i + 1]) : "r"(b), "r"(two_to_e));
                }
                // V rows past the sequence's end may hold anything, and their weight of 0 does not make a NaN harmless
                if (kv == 1 && key + key7 >= valid) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = 0u;
                }
                unsigned char* to = dst + (j >> 1) * 2048 + (j & 1) * 1024;
                *reinterpret_cast<uint4*>(to + (((2 * piece) ^ key7) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(to + (((2 * piece + 1) ^ key7) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&aux->full16[slot]));
                mbar_arrive(smem_u32(&aux->raw_empty[2u * place + kv]));
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ kernel
// kManySeqs, kWide as in verify_attn_umma_kernel; kF16: q and out are fp16 instead of bf16.
template <bool kManySeqs, bool kWide, bool kF16>
__global__ void __launch_bounds__(kFp8Threads, 1)
verify_attn_fp8_kernel(const AttnParams p, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ __align__(1024) unsigned char smem[];
    AuxFp8* aux = reinterpret_cast<AuxFp8*>(smem + kAuxOff);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem_base = smem_u32(smem);
    if (smem_base & 1023u) {                       // operand tiles must sit on swizzle-atom boundaries
        if (tid == 0) report(p.status, kErrTimeout);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < kFp8Slots; ++i) {
            mbar_init(smem_u32(&aux->empty[i]), 1);
            mbar_init(smem_u32(&aux->full16[i]), 4);
        }
        for (int i = 0; i < kRawSlots<kWide>; ++i) {
            mbar_init(smem_u32(&aux->raw_full[i]), i & 1 ? 1 : 2);      // the bytes, and for a tile's K slot the note
            mbar_init(smem_u32(&aux->raw_empty[i]), 4);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&aux->s_full[s]), 1);
            mbar_init(smem_u32(&aux->o_done[s]), 1);
        }
        mbar_init(smem_u32(&aux->q_full), 256);
        for (int i = 0; i < kSegs; ++i) mbar_init(smem_u32(&aux->seg_full[i]), 1);
        aux->abort_flag = 0;
        aux->seg_reached = 0;
        aux->seg_close = 0x7fffffff;
        aux->seg_bad_tree = 0;
        aux->sched_b0 = 0; aux->sched_tile_begin = 0;
        fence_barrier_init();
        tma_prefetch_desc(&kmap);
        tma_prefetch_desc(&vmap);
    }
    if (warp == 0) { tmem_alloc(smem_u32(&aux->tmem_base), kTmemCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = aux->tmem_base;
    if (warp == 2) {                               // (as in verify_attn_umma_kernel)
        const long long line = 32ll * blockIdx.x + lane;
        if (line * 128 < (long long)p.batch * p.max_pages_per_seq * 4) l2_prefetch(reinterpret_cast<const char*>(p.block_table) + line * 128);
        if (lane * 32 < p.batch) {
            l2_prefetch(p.ctx_lens + lane * 32);
            if (p.node_offsets) l2_prefetch(p.node_offsets + lane * 32);
        }
        if (lane * 32 < p.total_nodes) l2_prefetch(p.tree_parent + lane * 32);
    }
    auto wait_for_inputs = [] {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    };
    Walker<kManySeqs> w;
    if constexpr (kManySeqs) {
        wait_for_inputs();
        build_walk<kFp8Threads>(p, aux, w);
    }
    // 128 x 72 + 128 x 80 + 256 x 176 = 64512 of the 512 x 128 registers that the CTA was launched with
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (!kManySeqs) wait_for_inputs();
        if (warp == 0) {
            if constexpr (!kManySeqs) build_walk_small(p, w);
            producer_loop_fp8<kWide, kManySeqs>(p, &kmap, &vmap, aux, smem_base + kRawOff<kWide>, w);
        } else if (warp == 1) {
            mma_loop<kWide, true, true>(aux, smem_base, tmem);
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (!kManySeqs) wait_for_inputs();
        convert_loop<kWide>(p, aux, smem);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        if (!kManySeqs) wait_for_inputs();
        softmax_loop<kWide, kF16, true>(p, aux, smem, tmem, warp >= 8 ? 1 : 0);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        if (aux->abort_flag) {
            // (as in verify_attn_umma_kernel: copies may still be in flight)
            const uint64_t t0 = global_timer_ns();
            for (int polls = 0; polls < (1 << 22) && global_timer_ns() - t0 < 2000000ull; ++polls) {}
            if (lane == 0) report(p.status, kErrTimeout);
        }
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

}  // namespace umma_path
}  // namespace owl
