// Verify attention over the 8-bit cache (fp8_block.cuh).  Partition, segments, partials and the order of events are those of
// verify_attn_umma.cuh; what differs follows from K and V arriving as e4m3.
//
//   S = Q K^T   on 8-bit operands, K straight from where TMA put it.  A row of Q, divided by a power of two, is cut into e4m3 pieces, each
//               the remainder of those before: two for bf16 queries (eight significant bits, four a piece), three for fp16 ones.
//               The pieces' products add up in one accumulator.  What the pieces leave of an element is below half of e4m3's smallest step,
//               2^-10, where the row's largest element is above 224: 2^-17.8 of that largest element.  A block's 2^e multiplies its
//               columns of S, along with sm_scale, in fp32.
//   O += P V    on fp16 operands: four warps turn a V tile into fp16, 2^e included (exact but for what lies below fp16's smallest
//               step, 2^-24), and the weights are fp16.  Weights cut into e4m3 pieces would lose what is below 2^-15 of the largest, which
//               is where a long context's mass may lie beside one dominant key.
//
// Two e4m3 products of 128x128x32 take the time of one fp16 pair, so the tensor pipe does the work of the 16-bit caches' pass; HBM brings half
// of its bytes, and shared memory carries per tile 32 KB from TMA, 64 for Q K^T, 16 + 32 for the conversion and 32 for P V.  (A
// form that turned K into fp16 as well moved 224 KB, kept the ring half as deep, and took 453 us on 16 chains of 8 at 4K to 64K, where
// this one takes 283 to 305.)
// What bounds it: no unit of an SM alone.  A tile of a chain takes some 2300 clocks, of which HBM needs 1370 at the copy bandwidth, the softmax
// warps work 970 (and wait 510 for the product two tiles back) and the converting warps 1310 (and wait 670 for their slot and 500 for V): the
// ring of these is what a tile takes; 16 chains run at 4.0 TB/s, 62 % of the copy bandwidth.  16 trees of 32, 128 rows a unit, take 1700 clocks a
// tile, 1024 of them exponentials at 16 ex2 a clock.  One tree of 32 at 32K (31 to 33 us) is 14 such tiles a CTA, 12 us, 10 us of
// start and merge, and some 10 us that are not accounted for; a chain at 2K (13 us) is set-up, first copies and the merge.
// Back to back the long cases also meet the board's 1000 W.  One GPU, a pass alone / back to back and its SM clock: 16 chains 305 / 302 us
// at 1.85 GHz, 16 mixed 338 / 387 at 1.78, 16 trees of 32 350 / 399 at 1.53, 4 x 64K of fp16 342 / 362 at 1.63 (of 1.965 GHz).
// The instances for wide units spill: 28 to 112 bytes of stores and 32 to 340 of loads at 176 registers for the softmax warps, those for
// narrow ones 0 to 4 and 0 to 44.
//
// 16 warps:
//   warp 0        TMA producer: one box per (page, head) of K and of V into a ring of tiles of 2 x 16 KB; leaves each tile's note
//   warp 1        issues the products
//   warps 4-11    softmax, two streams
//   warps 12-15   turn V into fp16, two slots of 32 KB
//
// Units of more than 128 rows ("shared"): two streams of 128 rows on the same tiles, each with its S, P and O in tensor memory, as in
// verify_attn_umma.cuh.
// Other units ("joint"): both softmax warpgroups work on each tile, one O, and three S, so that Q K^T runs up to three tiles ahead and no
// softmax waits for the products of the tile before.  (With two streams that took the tiles by turns, each waiting for its own
// P V and Q K^T, a 128-row tile took 2100 clocks: 16 chains of 64-row units 411 us, now 312 to 360.)
//   65 to 128 rows: rows on the lanes, each warpgroup weighs half of a tile's keys; the two share the rows' references.
//   up to 64 rows:  keys on the lanes.  The products are turned round,
//       S^T = K Q^T   [128 keys x pieces * rows], the pieces' columns added up in registers,
//       O^T += V^T P  [128 channels x rows],      P [keys x rows] through shared memory,
//     so that a unit of 32 rows does not pay for 128 of them: the products take an eighth and a quarter of the multipliers (and of the
//     power, which sets the clock where calls follow each other), a softmax thread has one key and half of the rows, every lane is in use, and sums
//     over keys are kept per thread until the segment's end.
#pragma once

#include "fp8_block.cuh"
#include "verify_attn_umma.cuh"

namespace owl {
namespace umma_path {

constexpr int kFp8Threads = 512;
constexpr int kPieceBytes = 128 * kHeadDim;          // 16 KB: one piece of 128 rows of Q; also a raw K or V tile
constexpr int kFp8VSlots = 2;                        // fp16 V tiles, 32 KB each
constexpr int kNotes = 8;
constexpr int kPartialRows = kRows;                  // (`kRows` below is also a constant of a template)
constexpr int kKeysRows = 64;                        // most rows of a unit with its keys on the lanes
constexpr int kPBytes = kTileKeys * 128;             // its P: 128 bytes (64 rows) per key, one per stream
// Shared memory: Q (its pieces; keys on lanes: fewer rows, then the two P), the fp16 V tiles, the ring of raw tiles, scratch.
template <bool kF16> constexpr int kPieces = kF16 ? 3 : 2;
template <bool kF16> constexpr int kPOff = kPieces<kF16> * kKeysRows * kHeadDim;
constexpr int larger(int a, int b) { return a > b ? a : b; }
template <bool kWide, bool kF16> constexpr int kVOff = larger((kWide ? 2 : 1) * kPieces<kF16> * kPieceBytes, kPOff<kF16> + 2 * kPBytes);
template <bool kWide, bool kF16> constexpr int kRawOff = kVOff<kWide, kF16> + kFp8VSlots * kSlotBytes;
template <bool kWide, bool kF16> constexpr int kRawTiles = (kAuxOff - kRawOff<kWide, kF16>) / (2 * kPieceBytes);
static_assert(kRawTiles<false, false> == 3 && kRawTiles<false, true> == 3 && kRawTiles<true, false> == 3 && kRawTiles<true, true> == 2, "layout");
// Joint units' numbers of their rows.
struct KeysScratch {
    float scale[kKeysRows], bias[kKeysRows];         // a weight is exp2(score * scale + bias)
    float m[kKeysRows], alpha[kKeysRows];
    unsigned most[4][kKeysRows];                     // largest score of the tile by warp, as an ordered integer
    float sum[4][kKeysRows];                         // of the weights, by warp
    float w[kKeysRows];                              // what O is multiplied by
};
struct RowsScratch {
    float most[2][128], sum[2][128];                 // by warpgroup
};
static_assert(sizeof(RowsScratch) <= sizeof(KeysScratch), "the larger one is counted");
template <bool kWide, bool kF16> constexpr int kScratchOff = kWide ? kPOff<kF16> + 2 * kPBytes : kRawOff<kWide, kF16> + kRawTiles<kWide, kF16> * 2 * kPieceBytes;
static_assert(kScratchOff<false, false> + sizeof(KeysScratch) <= kAuxOff && kScratchOff<false, true> + sizeof(KeysScratch) <= kAuxOff, "layout");
static_assert(kScratchOff<true, false> + sizeof(KeysScratch) <= kVOff<true, false> && kScratchOff<true, true> + sizeof(KeysScratch) <= kVOff<true, true>, "layout");
// Tensor memory: shared S0 S1 O0 O1 of 128 columns; joint three S of 128 columns (two of 192: fp16, 64 rows, keys on lanes) and O.
constexpr uint32_t kJointO = 384;
__device__ __forceinline__ uint32_t joint_buffers(uint32_t columns) { return columns > 128u ? 2u : 3u; }
__device__ __forceinline__ uint32_t joint_s(uint32_t buffer, uint32_t columns) { return buffer * (columns > 128u ? 192u : 128u); }

// What is known of a tile besides its bytes.  A place is written again eight tiles later: the producer is at most kRawTiles ahead of
// Q K^T, and that at most three tiles ahead of the softmax warps, the last to look at it.
struct TileNote {
    float kscale[kTileKeys / 16];                // 2^(e + 24) of K, for each 16 keys (score_scale)
    int spans;                                   // low half: keys of the sequence in it (-1: no more tiles); high: of them, the context's
    int8_t vexp[kTileKeys / 16];                 // e of V
};
struct AuxFp8 : Aux {
    uint64_t raw_full[6], raw_empty[6];          // K and V of each raw tile
    uint64_t v_full[kFp8VSlots], v_empty[kFp8VSlots];
    uint64_t joint_s_full[3], joint_o_done;
    TileNote note[kNotes];
    uint8_t nan_drafts[kNotes];                  // of the tile: a drafted row of V has a NaN, which its fp16 tile has not
    float row_scale[kRows];                      // what the rows of Q were divided by
};
static_assert(sizeof(AuxFp8) <= kAuxBytes, "aux area too small");
static_assert(kNotes > 3 + 3, "a note outlives its tile's place in the ring");

// Rows that a unit with its keys on the lanes is padded to; 0: its rows are on the lanes.
__device__ __forceinline__ int keys_rows(int M) { return M <= 32 ? 32 : M <= kKeysRows ? 64 : 0; }
// Warps of a stream's warpgroup with something to do in a unit of up to 128 rows.
__device__ __forceinline__ int live_warps_fp8(int M) { return M <= kKeysRows ? 4 : (M + 31) >> 5; }

// ------------------------------------------------------------------------------------------ producer
template <bool kWide, bool kF16, bool kManySeqs>
__device__ __forceinline__ void producer_loop_fp8(const AttnParams& p, const CUtensorMap* kmap, const CUtensorMap* vmap, AuxFp8* aux,
                                                  uint32_t raw, Walker<kManySeqs> w) {
    constexpr uint32_t kPlaces = kRawTiles<kWide, kF16>;
    const int lane = threadIdx.x & 31;
    volatile int* abort_flag = &aux->abort_flag;
    const int ppt = kTileKeys >> p.page_shift;               // pages (= TMA boxes) per tile
    const int block_tiles = 32 / ppt;
    const uint32_t box_bytes = (uint32_t)p.page_size * 128u;
    const int oob = p.num_pages * p.num_kv_heads;            // a coordinate past the end: the box reads zeros
    const uint64_t stream_policy = l2_policy_evict_first();
    uint32_t place = 0, free_parity = 1, seq = 0;
    for (uint32_t seg_no = 0;; ++seg_no) {
        Segment g;
        g.b = g.n = g.L = 0;
        const bool more = w.template next<kWide>(p, g);
        const int keys = g.L + g.n;
        const int pages_valid = (keys + p.page_size - 1) >> p.page_shift;
        const int32_t* table = p.block_table + (long long)g.b * p.max_pages_per_seq;
        // 32 pages of the table at a time, one per lane: those of the tiles from `t` on.  Pages are asked for two such blocks ahead and their
        // exponents (K's in the low byte, V's in the high one) one block ahead, which is four tiles with the smallest pages: an
        // exponent is a load that waits for a load.
        auto pages_of = [&](int t) {
            const int lp = t * ppt + lane;
            return t < g.tile1 && lp < pages_valid ? table[lp] : -1;
        };
        auto exps_of = [&](int pg) -> int {
            return (unsigned)pg < (unsigned)p.num_pages ? *reinterpret_cast<const uint16_t*>(p.page_exp + ((long long)pg * p.num_kv_heads + g.h) * 2) : 0;
        };
        int pages = more ? pages_of(g.tile0) : -1, pages_next = more ? pages_of(g.tile0 + block_tiles) : -1;
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
        int exps = 0, exps_next = 0, pages_after = -1;
        for (int t = g.tile0, in_block = 0; t < g.tile1; ++t) {
            const int page = __shfl_sync(0xffffffffu, pages, in_block * ppt + lane);      // of the tile's pages, this lane's (lanes below ppt)
            int coord = oob;
            if ((unsigned)page < (unsigned)p.num_pages) coord = page * p.num_kv_heads + g.h;
            else if (lane < ppt && t * ppt + lane < pages_valid) {
                report(p.status, kErrBadPage);
                const_cast<volatile int&>(announced.bad_page) = 1;
            }
            bool ok = true;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const uint32_t slot = 2u * place + kv, full = smem_u32(&aux->raw_full[slot]);
                // (one verdict for the warp: its lanes go on together)
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&aux->raw_empty[slot]), free_parity, abort_flag)) && ok;
                if (ok && lane == 0) mbar_arrive_expect_tx(full, (uint32_t)kPieceBytes);
                __syncwarp();
                if (ok && lane < ppt)
                    tma_load_3d_hint(raw + slot * kPieceBytes + lane * box_bytes, kv ? vmap : kmap, full, 0, 0, coord, stream_policy);
                __syncwarp();
            }
            // (asked for after the tile's copies: the segment's first copies are what a short call waits for)
            if (t == g.tile0) exps = exps_of(pages);
            if (in_block == 0) {
                exps_next = exps_of(pages_next);
                pages_after = pages_of(t + 2 * block_tiles);
            }
            // the note: an arrival of its own on both barriers
            TileNote& note = aux->note[seq % kNotes];
            const int exp_kv = __shfl_sync(0xffffffffu, exps, in_block * ppt + ((lane * 16) >> p.page_shift));
            if (lane < kTileKeys / 16) {
                note.kscale[lane] = exp2_int(max(kExpMin, min(kExpMax, (int)(int8_t)(exp_kv & 0xff))) - kExpMin);
                note.vexp[lane] = (int8_t)(exp_kv >> 8);
            }
            if (lane == 0) {
                note.spans = min(kTileKeys, keys - t * kTileKeys) | max(0, min(kTileKeys, g.L - t * kTileKeys)) << 16;
                aux->nan_drafts[seq % kNotes] = 0;
            }
            __syncwarp();
            if (lane < 2) mbar_arrive(smem_u32(&aux->raw_full[2u * place + lane]));
            if (++in_block == block_tiles) { in_block = 0; pages = pages_next; exps = exps_next; pages_next = pages_after; }
            if (++place == kPlaces) { place = 0; free_parity ^= 1u; }
            ++seq;
        }
    }
    // no more tiles (after a wait that gave up the converting warps stop by themselves)
    const bool ok = mbar_wait(smem_u32(&aux->raw_empty[2u * place + 1u]), free_parity, abort_flag);
    if (lane == 0 && ok) {
        aux->note[seq % kNotes].spans = -1;
        mbar_arrive(smem_u32(&aux->raw_full[2u * place + 1u]));
        mbar_arrive(smem_u32(&aux->raw_full[2u * place + 1u]));
    }
}

// ------------------------------------------------------------------------------------------ V to fp16
// Warp w of four takes key groups 4w .. 4w + 3 of a tile, eight keys x 64 elements per turn `j`.  Lane: 16 elements (one 16-byte piece) of
// one key.  Raw rows are 128 bytes with piece x at place x ^ (key & 7), operand rows 128 bytes per half of the head dimension with
// piece y at y ^ (key & 7), and a raw piece becomes operand pieces 2x, 2x + 1: eight neighbouring lanes take four pieces of two keys
// that differ in bits 0 and 2, so that neither the loads nor the stores meet in a bank.
__device__ __forceinline__ uint4 load_v(const unsigned char* src, int j, int piece, int key7) {
    return *reinterpret_cast<const uint4*>(src + (j >> 1) * 1024 + ((((j & 1) * 4 + piece) ^ key7) << 4));
}
__device__ __forceinline__ void convert_v(const uint4& u, int j, const TileNote& note, int warp, unsigned char* dst, int piece, int key7) {
    const int e = max(kExpMin, min(kExpMax, (int)note.vexp[2 * warp + (j >> 2)]));
    const uint32_t one = e >= -14 ? (uint32_t)(e + 15) << 10 : 1u << (e + 24);
    const uint32_t two_to_e = one | one << 16;
    uint32_t o[8];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = e4m3x2_to_f16x2(w[i] & 0xffffu), b = e4m3x2_to_f16x2(w[i] >> 16);
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * i]) : "r"(a), "r"(two_to_e));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * i + 1]) : "r"(b), "r"(two_to_e));
    }
    unsigned char* to = dst + (j >> 1) * 2048 + (j & 1) * 1024;
    *reinterpret_cast<uint4*>(to + (((2 * piece) ^ key7) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(to + (((2 * piece + 1) ^ key7) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
}
__device__ __forceinline__ uint32_t drop_nans(uint32_t& v) {
    const uint32_t nans = __vcmpeq4(v & 0x7f7f7f7fu, 0x7f7f7f7fu);
    v &= ~nans;
    return nans;
}
template <bool kWide, bool kF16>
__device__ __forceinline__ void convert_loop(const AttnParams& p, AuxFp8* aux, unsigned char* smem) {
    constexpr uint32_t kPlaces = kRawTiles<kWide, kF16>;
    constexpr unsigned kAll = 0xffffffffu;
    volatile int* abort_flag = &aux->abort_flag;
    const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
    const int r = lane >> 2, key7 = (r >> 1) ^ ((r & 1) * 5), piece = lane & 3;
    const unsigned char* raw = smem + kRawOff<kWide, kF16> + kPieceBytes + warp * 4096 + key7 * 128;
    unsigned char* ring = smem + kVOff<kWide, kF16> + warp * 8192 + key7 * 128;
    uint32_t place = 0, parity = 0;
    for (uint32_t n = 0;; ++n) {
        if (!__all_sync(kAll, mbar_wait(smem_u32(&aux->raw_full[2u * place + 1u]), parity, abort_flag))) return;
        const TileNote& note = aux->note[n % kNotes];
        const int spans = const_cast<const volatile int&>(note.spans), valid = (int16_t)(spans & 0xffff), context = spans >> 16;
        if (valid < 0) return;
        const uint32_t slot = n % kFp8VSlots;
        if (!__all_sync(kAll, mbar_wait(smem_u32(&aux->v_empty[slot]), ((n / kFp8VSlots) & 1u) ^ 1u, abort_flag))) return;
        const unsigned char* src = raw + 2u * place * kPieceBytes;
        unsigned char* dst = ring + slot * kSlotBytes;
        if (__builtin_expect(context >= valid, 1)) {      // the context's keys alone, all of the tile
            uint4 u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = load_v(src, j, piece, key7);
#pragma unroll
            for (int j = 0; j < 8; ++j) convert_v(u[j], j, note, warp, dst, piece, key7);
        } else {
            // A tile that holds drafted rows, or ends.  Rows past the sequence's end may hold anything, and their weight of 0 does not make a
            // NaN harmless; nor does it that of a drafted row in the rows of Q that do not see its node: such NaNs are left out, and those that
            // do see it get them at the segment's end (mark_nan_drafts).  Apart from the other tiles, and short: with this looked at in
            // every tile 16 mixed sequences of 4K to 64K took 468 us, unrolled by two in the loop's middle 360, like this 340 on the same GPU
            // (from one GPU to the next 312 to 390).
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                const int key = (4 * warp + (j >> 1)) * 8 + key7;
                uint4 u = load_v(src, j, piece, key7);
                if (key >= valid) u = make_uint4(0u, 0u, 0u, 0u);
                else if (key >= context && (drop_nans(u.x) | drop_nans(u.y) | drop_nans(u.z) | drop_nans(u.w)))
                    const_cast<volatile uint8_t&>(aux->nan_drafts[n % kNotes]) = 1;
                convert_v(u, j, note, warp, dst, piece, key7);
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(smem_u32(&aux->v_full[slot]));
            mbar_arrive(smem_u32(&aux->raw_empty[2u * place + 1u]));
        }
        if (++place == kPlaces) { place = 0; parity ^= 1u; }
    }
}

// ------------------------------------------------------------------------------------------ MMA issuer
// K arrives in the raw ring, V apart from it as an fp16 tile.  In shared units the softmax warp that looks at the next K tile for this warp
// also makes sure of V before it announces P.
template <bool kWide, bool kF16>
__device__ __forceinline__ void mma_loop_fp8(AuxFp8* aux, uint32_t smem_base, uint32_t tmem) {
    constexpr unsigned kAll = 0xffffffffu;
    constexpr uint32_t kPlaces = kRawTiles<kWide, kF16>;
    volatile int* abort_flag = &aux->abort_flag;
    constexpr uint32_t idesc_qk = umma_idesc_e4m3(128, kTileKeys);
    constexpr uint32_t idesc_pv = umma_idesc_16bit(128, kHeadDim, 0, 1, true);
    const uint32_t elected = elect_one() ? 1u : 0u;
    // of Q's first piece, of the first raw K tile and of the first V tile; the others differ in the start address
    const uint64_t q_desc0 = umma_smem_desc_sw128(smem_base, 16, 1024);
    const uint64_t k_desc0 = umma_smem_desc_sw128(smem_base + kRawOff<kWide, kF16>, 16, 1024);
    const uint64_t v_desc0 = umma_smem_desc_sw128(smem_base + kVOff<kWide, kF16>, 1024, 2048);
    const uint32_t q_hi = (uint32_t)(q_desc0 >> 32), k_hi = (uint32_t)(k_desc0 >> 32), v_hi = (uint32_t)(v_desc0 >> 32);
    const uint32_t raw_full = smem_u32(&aux->raw_full[0]), raw_empty = smem_u32(&aux->raw_empty[0]);
    const uint32_t v_full = smem_u32(&aux->v_full[0]), v_empty = smem_u32(&aux->v_empty[0]);
    const uint32_t s_full = smem_u32(&aux->s_full[0]), o_done = smem_u32(&aux->o_done[0]), joint_s_full = smem_u32(&aux->joint_s_full[0]);
    uint32_t seg_no = 0, k_place = 0, k_parity = 0, v_seq = 0;

    auto qk = [&](uint32_t issue, uint32_t tS, uint32_t q_lo) {
        const uint32_t k_lo = (uint32_t)k_desc0 + k_place * (uint32_t)(2 * kPieceBytes >> 4);
#pragma unroll
        for (int piece = 0; piece < kPieces<kF16>; ++piece)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                umma_f8_ss_lh_if(issue, tS, q_lo + (uint32_t)((piece * kPieceBytes + ks * 32) >> 4), q_hi, k_lo + (uint32_t)(ks * 32 >> 4), k_hi,
                                 idesc_qk, (piece | ks) ? 1u : 0u);
    };
    auto pv = [&](uint32_t issue, uint32_t tS, uint32_t accumulate) {
        const uint32_t v_lo = (uint32_t)v_desc0 + (v_seq % kFp8VSlots) * (uint32_t)(kSlotBytes >> 4);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
            umma_ts_lh_if(issue, tS + 256, tS + ks * 8, v_lo + (uint32_t)(ks * 4096 >> 4), v_hi, idesc_pv, ks ? 1u : accumulate);
    };
    // joint units; `keys`: keys on lanes, the padded rows
    const uint64_t p_desc0 = umma_smem_desc_sw128(smem_base + kPOff<kF16>, 1024, 1024);
    auto qk_joint = [&](uint32_t issue, uint32_t tS, uint32_t keys) {
        if (!keys) { qk(issue, tS, (uint32_t)q_desc0); return; }
        const uint32_t k_lo = (uint32_t)k_desc0 + k_place * (uint32_t)(2 * kPieceBytes >> 4);
        const uint32_t idesc = umma_idesc_e4m3(128, 0) | (kPieces<kF16> * keys >> 3) << 17;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
            umma_f8_ss_lh_if(issue, tS, k_lo + (uint32_t)(ks * 32 >> 4), k_hi, (uint32_t)q_desc0 + (uint32_t)(ks * 32 >> 4), q_hi, idesc, ks ? 1u : 0u);
    };
    auto pv_joint = [&](uint32_t issue, uint32_t tP, uint32_t i, uint32_t keys) {
        const uint32_t v_lo = (uint32_t)v_desc0 + (v_seq % kFp8VSlots) * (uint32_t)(kSlotBytes >> 4), acc0 = i > 0 ? 1u : 0u;
        if (!keys) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_ts_lh_if(issue, tmem + kJointO, tP + ks * 8, v_lo + (uint32_t)(ks * 4096 >> 4), v_hi, idesc_pv, ks ? 1u : acc0);
            return;
        }
        const uint32_t p_lo = (uint32_t)p_desc0 + (i & 1u) * (uint32_t)(kPBytes >> 4), p_hi = (uint32_t)(p_desc0 >> 32);
        const uint32_t idesc = umma_idesc_16bit(128, 0, 1, 1, true) | keys >> 3 << 17;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
            umma_ss_lh_if(issue, tmem + kJointO, v_lo + (uint32_t)(ks * 4096 >> 4), v_hi, p_lo + (uint32_t)(ks * 2048 >> 4), p_hi, idesc, ks ? 1u : acc0);
    };
    auto next_k = [&] { if (++k_place == kPlaces) { k_place = 0; k_parity ^= 1u; } };

    for (;;) {
        meet_before_segment(aux, seg_no, false);
        const Segment g = announced_segment(aux, seg_no);
        const int tile0 = __reduce_max_sync(kAll, g.tile0), tile1 = __reduce_max_sync(kAll, g.tile1);
        if (tile1 == 0) break;
        const bool shared = kWide && __reduce_max_sync(kAll, g.shared ? 1 : 0) != 0;
        bool ok = __all_sync(kAll, mbar_wait(smem_u32(&aux->q_full), seg_no & 1u, abort_flag));
        const int T = tile1 - tile0;
        ++seg_no;
        if (!shared) {
            const uint32_t keys = (uint32_t)__reduce_max_sync(kAll, keys_rows(g.M)), columns = keys ? kPieces<kF16> * keys : 128u;
            const int p_threads = 32 + 64 * __reduce_max_sync(kAll, live_warps_fp8(g.M)), ahead = (int)joint_buffers(columns);
            uint32_t b = 0, p_bar = 0;              // S buffer of the tile; hardware barrier of its P, 9 + p_bar
            // S = Q K^T of the segment's next tile, announced on every path (mma_loop says why)
            auto next_s = [&] {
                ok = __all_sync(kAll, mbar_wait(raw_full + k_place * 16u, k_parity, abort_flag)) && ok;
                tc_fence_after();
                const uint32_t issue = ok ? elected : 0u;
                qk_joint(issue, tmem + joint_s(b, columns), keys);
                umma_commit_if(issue, joint_s_full + b * 8u);
                if (!ok && elected) mbar_arrive(joint_s_full + b * 8u);
                umma_commit_if(issue, raw_empty + k_place * 16u);
                next_k();
            };
            for (int i = 0; i < ahead && i < T; ++i) { b = (uint32_t)i; next_s(); }
            b = 0;
#pragma unroll 1
            for (int i = 0; i < T; ++i) {
                // V is looked at while P is being made; then P is announced on hardware barrier 9, 10 or 11, each every third tile: a warp
                // that arrives for tile i + 3 has seen its S, which is issued after this warp's bar.sync for tile i (so one
                // generation never sees two tiles' arrivals)
                ok = __all_sync(kAll, mbar_wait(v_full + (v_seq % kFp8VSlots) * 8u, (v_seq / kFp8VSlots) & 1u, abort_flag)) && ok;
                asm volatile("bar.sync %0, %1;" ::"r"(9 + p_bar), "r"(p_threads) : "memory");
                tc_fence_after();
                const uint32_t issue = ok ? elected : 0u;
                pv_joint(issue, tmem + joint_s(b, columns), (uint32_t)i, keys);
                umma_commit_if(issue, v_empty + (v_seq % kFp8VSlots) * 8u);
                if (i == T - 1) {
                    umma_commit_if(issue, smem_u32(&aux->joint_o_done));
                    if (!ok && elected) mbar_arrive(smem_u32(&aux->joint_o_done));
                }
                ++v_seq;
                // the product that reads this tile's P has been issued: its S buffer takes the tile `ahead` tiles on
                if (i + ahead < T) next_s();
                if (++b == (uint32_t)ahead) b = 0;
                if (++p_bar == 3u) p_bar = 0;
            }
            continue;
        }
        if constexpr (kWide) {
            // two streams of 128 rows on the same tiles: mma_loop's turns
#pragma unroll 1
            for (int i = -1; i < T; ++i) {
                const bool do_pv = i >= 0, do_qk = i + 1 < T;
                const uint32_t v_bar = v_empty + (v_seq % kFp8VSlots) * 8u, k_bar = raw_empty + k_place * 16u;
                uint32_t q_lo = (uint32_t)q_desc0, tS = tmem;
                if (i < 0) ok = __all_sync(kAll, mbar_wait(raw_full + k_place * 16u, k_parity, abort_flag)) && ok;
                tc_fence_after();
                const uint32_t issue = ok ? elected : 0u;
#pragma unroll 1
                for (uint32_t s = 0; s < 2; ++s) {
                    if (do_pv) {
                        // P of the tile (and that V has been turned into fp16) is announced on hardware barrier 4 + s
                        asm volatile("bar.sync %0, 160;" ::"r"(4 + s) : "memory");
                        tc_fence_after();
                        pv(issue, tS, i > 0 ? 1u : 0u);
                        umma_commit_if(s ? issue : 0u, v_bar);
                        umma_commit_if(do_qk ? 0u : issue, o_done + s * 8u);
                        if (!ok && !do_qk && elected) mbar_arrive(o_done + s * 8u);
                    }
                    if (do_qk) {
                        if (do_pv && s == 0) asm volatile("bar.sync 6, 64;" ::: "memory");      // the next K tile has landed
                        qk(issue, tS, q_lo);
                        umma_commit_if(issue, s_full + s * 8u);
                        if (!ok && elected) mbar_arrive(s_full + s * 8u);
                        umma_commit_if(s ? issue : 0u, k_bar);
                    }
                    tS += 128; q_lo += (uint32_t)(kPieces<kF16> * kPieceBytes >> 4);
                }
                if (do_pv) ++v_seq;
                if (do_qk) next_k();
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ softmax warpgroups
// Q rows to e4m3 pieces in shared memory, rows of 128 bytes (K-major, 128-byte swizzle); rows beyond M are zeros.  A thread has eight elements
// (piece `c` of sixteen) of every eighth row, `count` rows from packed row `row` on; `dst`: the row's place in the first piece, the
// next piece's lies `piece_bytes` on.
template <bool kF16>
__device__ __forceinline__ void load_q_fp8(const AttnParams& p, const Segment& g, AuxFp8* aux, unsigned char* dst, const int piece_bytes, int row,
                                           const int count, const int c) {
    const int G = p.group;
    dst += ((c >> 1) ^ (row & 7)) * 16 + (c & 1) * 8;
#pragma unroll 1
    for (int j0 = 0; j0 < count; j0 += 4) {
        uint4 u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned r = (unsigned)(row + 8 * j), node = row_node(p, r);
            const __nv_bfloat16* src = p.q + ((long long)(g.node_base + node) * p.num_q_heads + g.h * G + (r - node * G)) * kHeadDim + c * 8;
            u[j] = j0 + j < count && r < (unsigned)g.M ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j0 + j >= count) break;
            const uint32_t w[4] = {u[j].x, u[j].y, u[j].z, u[j].w};
            float x[8];
            uint32_t most = 0u;                        // bits of the largest magnitude; a NaN's are larger than any
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (kF16) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    x[2 * i] = f.x; x[2 * i + 1] = f.y;
                } else {
                    x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                }
                most = max(most, max(__float_as_uint(x[2 * i]) & 0x7fffffffu, __float_as_uint(x[2 * i + 1]) & 0x7fffffffu));
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
            // the smallest power of two with (largest magnitude) <= 448 of them (block_exponent, over the types' range)
            const int e = max(-110, min(120, (int)((most + 0x1fffffu) >> 23) - 135));
            const float inv = exp2_int(-e);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
#pragma unroll
            for (int piece = 0; piece < kPieces<kF16>; ++piece) {
                const uint2 v = make_uint2(pack_e4m3x4(y[0], y[1], y[2], y[3]), pack_e4m3x4(y[4], y[5], y[6], y[7]));
                *reinterpret_cast<uint2*>(dst + piece * piece_bytes) = v;
                if (piece + 1 < kPieces<kF16>) {
                    const float4 a = e4m3x4_to_f32(v.x), b = e4m3x4_to_f32(v.y);
                    y[0] -= a.x; y[1] -= a.y; y[2] -= a.z; y[3] -= a.w; y[4] -= b.x; y[5] -= b.y; y[6] -= b.z; y[7] -= b.w;
                }
            }
            // (a row with an infinity or a NaN has no pieces: its scores are NaN, and so is what comes of them)
            if (c == 0) aux->row_scale[row + 8 * j] = most >= 0x7f800000u ? __int_as_float(0x7fffffff) : exp2_int(e);
            dst += 1024;
        }
        row += 32;
    }
}

// Weights are kept 2^7 above exp2(score - m), up to 2^15, so that fp16 (largest 65504, smallest step 2^-24) holds what is 2^-31 of the
// reference.  The normaliser sums them as they are, not as fp16 rounds them: that is off by at most 2^-12 of the output, where one
// key has all the weight, and two conversions and an addition per pair of keys less (8 trees of 32 at 64K, 64 query heads: 647 -> 592 us).
constexpr float kWeightShift = 7.f;
constexpr float kWeightLimit = 32768.f;          // 2^(8 + 7)
constexpr float kNoReference = 3.402823466e38f;  // in the place of 7 - m: takes any score above -inf beyond the limit
// log-sum-exp of a row from its reference and its sum of shifted weights (a NaN sum stays one)
__device__ __forceinline__ float lse_of_sum(float m, float sum) {
    return sum > 0.f ? (m - kWeightShift + __log2f(sum)) * 0.6931471805599453f : sum == 0.f ? -INFINITY : sum;
}
__device__ __forceinline__ unsigned ordered(float x) {        // sorts like x; a NaN is below everything
    const unsigned u = __float_as_uint(x);
    return x != x ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(unsigned u) { return u == 0u ? -INFINITY : __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ float min_or_nan(float x, float y) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
// What a row's sums of products are multiplied by, besides their page's 2^(e + 24).  (The 2^24 keep the product of a row near the end of bf16's
// range finite that the page's 2^e brings back.)  Not below 2^-124, where all that is less makes scores that differ by less than 2^-66: times
// the smallest page's 1 it is no zero, and a score of -inf stays one.  (A NaN stays one, too.)
__device__ __forceinline__ float score_scale(const AttnParams& p, float row_scale) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(p.sm_scale * (1.4426950408889634f * exp2_int(kExpMin)) * row_scale), "f"(exp2_int(-124)));
    return r;
}
// A score is rounded before its reference is subtracted, in the weights as in the reference itself.  A product fused with the difference is
// not, and from references of this size on, whose neighbours lie further apart than 1, that makes the weight of the reference's own key
// anything from nothing to infinity.  Joint units multiply by the row's number, rounded, and then by the page's power of two, which is
// exact and may be fused.  Shared units fuse both while no row of the warp has a far reference (the joint units' form there: 4 x 64K of
// fp16 320 instead of 314 us, 8 x 64K of bf16 with 64 query heads 550 instead of 532).
constexpr float kFarReference = 16777216.f;
// Meets `count` threads on hardware barrier `id`; true for all if it is for one.
__device__ __forceinline__ bool any_of(int id, int count, bool mine) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %3, 0;\n\tbarrier.cta.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
                 : "=r"(r) : "r"(id), "r"(count), "r"(mine ? 1u : 0u) : "memory");
    return r != 0;
}

// What a segment's threads know of it, in either kind of joint unit.
struct JointSegment {
    const Segment& g;
    uint32_t tile_base, seg_no;      // the CTA's key tiles and segments so far
    bool leader;
};
// The product O += P V of key tile `seq` has completed.  (Its barrier's next phase is that of tile seq + 2, whose P has not been handed
// over.)
__device__ __forceinline__ void wait_for_product(AuxFp8* aux, uint32_t seq) {
    mbar_wait(smem_u32(&aux->v_empty[seq % kFp8VSlots]), (seq / kFp8VSlots) & 1u, &aux->abort_flag);
    __syncwarp();
    tc_fence_after();
}
// The softmax warps at a segment's end, its products awaited.  Whether the segment holds such drafted rows (they lie in the last two
// tiles of a sequence at most) is read by the first softmax warp alone and left for all before they meet, because a hardware barrier
// hangs on it: after a wait that gave up the converting and the producer warp may write the tiles' flags while others read them.
__device__ __forceinline__ void meet_at_segment_end(AuxFp8* aux, const JointSegment& js) {
    if (js.leader && (threadIdx.x & 31) == 0) {
        const volatile uint8_t* nans = aux->nan_drafts;
        const uint32_t T = (uint32_t)(js.g.tile1 - js.g.tile0), end = js.tile_base + T;
        const bool some = nans[(end - 1u) % kNotes] || (T > 1u && nans[(end - 2u) % kNotes]);
        const_cast<volatile int&>(aux->mark_drafts) = some && !*const_cast<volatile int*>(&aux->abort_flag);
    }
    meet_before_segment(aux, js.seg_no + 1, js.leader);
}
// S of the segment's tile i, in buffer `b`; `phases`: one bit per buffer, the phase of its barrier that comes next.
__device__ __forceinline__ void wait_for_scores(AuxFp8* aux, uint32_t b, uint32_t& phases) {
    mbar_wait_certain(smem_u32(&aux->joint_s_full[b]), (phases >> b) & 1u, &aux->abort_flag);
    phases ^= 1u << b;
    tc_fence_after();
}

// ------------------------------------------------------------------------------------------ joint units, rows on lanes
// Warpgroup s has the tile's keys [64 s, 64 s + 64); thread = row, in both.
template <bool kWide, bool kF16>
__device__ __forceinline__ void rows_segment(const AttnParams& p, AuxFp8* aux, unsigned char* smem, uint32_t tmem, const int s, const JointSegment& js,
                                             uint32_t& phases, const uint32_t done_phase) {
    const Segment& g = js.g;
    const int wtid = threadIdx.x - 128 - s * 128;
    const uint32_t lane_sel = (uint32_t)(((threadIdx.x >> 5) & 3) * 32) << 16;
    RowsScratch* k = reinterpret_cast<RowsScratch*>(smem + kScratchOff<kWide, kF16>);
    const int T = g.tile1 - g.tile0, rr = wtid, G = p.group;
    const int live = live_warps_fp8(g.M), both = 64 * live;      // threads of the two warpgroups that hold rows
    const bool idle = (wtid >> 5) >= live;
    const unsigned long long anc_row = rr < g.M ? aux->anc[row_node(p, rr)] : 0ull;
    const float scale2 = score_scale(p, aux->row_scale[rr]);
    float m = -INFINITY, l = 0.f;          // the row's reference, alike in both warpgroups; the sum over this one's keys
    uint32_t b = 0, p_bar = 0;
    for (int i = 0; i < (idle ? 0 : T); ++i) {
        const int t = g.tile0 + i;
        const uint32_t seq = js.tile_base + (uint32_t)i;
        wait_for_scores(aux, b, phases);
        const uint32_t tS = tmem + lane_sel + joint_s(b, 128u), tMine = tS + 64 * s;
        const float* kscale = aux->note[seq % kNotes].kscale + 4 * s;
        if ((t + 1) * kTileKeys > g.L) {
            // The tile reaches drafted positions (or the end of the sequence): at most two tiles per unit.
            // Visibility of this warpgroup's 64 keys for this row: prefix keys all, drafted key j iff ancestor-or-self.  The mask is
            // applied to S in tensor memory before the common path reads it.
            const int j0 = t * kTileKeys + 64 * s - g.L;
            const unsigned long long sees = j0 >= 64 ? 0ull : j0 >= 0 ? anc_row >> j0 : j0 <= -64 ? ~0ull : (~0ull >> (64 + j0)) | (anc_row << -j0);
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
                const uint32_t bits = (uint32_t)(sees >> (32 * c));
                uint32_t r[32];
                tmem_ld32(tMine + c * 32, r);
                tmem_wait_ld();
                tmem_loaded(r);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (!((bits >> j) & 1u)) r[j] = 0xff800000u;   // -inf
                tmem_st32(tMine + c * 32, r);
            }
            tmem_wait_st();
        }
        uint32_t pk[32];
        float sum;
        // up to three times: the references hold; some score was above its by more than the threshold; the first tile
        for (int tries = i == 0 ? 0 : 1;; ++tries) {
            if (tries != 1) {
                // the references move up to the tile's largest scores; the two warpgroups exchange theirs
                float mx = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    uint32_t r[32];
                    tmem_ld32(tMine + c * 32, r);
                    tmem_wait_ld();
                    tmem_loaded(r);
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        float a = __uint_as_float(r[16 * hf]);
#pragma unroll
                        for (int j = 1; j < 16; ++j) a = fmaxf(a, __uint_as_float(r[16 * hf + j]));
                        mx = fmaxf(mx, a * scale2 * kscale[2 * c + hf]);
                    }
                }
                k->most[s][wtid] = mx;
                named_barrier(8, both);
                const float m_new = fmaxf(m, fmaxf(mx, k->most[s ^ 1][wtid]));
                if (i > 0 && __any_sync(0xffffffffu, m_new > m)) {
                    const float alpha = m_new > m ? fast_exp2(m - m_new) : 1.f;
                    l *= alpha;
                    wait_for_product(aux, seq - 1u);
                    const uint32_t tO = tmem + lane_sel + kJointO + 64 * s;
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        uint32_t o[32];
                        tmem_ld32(tO + c * 32, o);
                        tmem_wait_ld();
                        tmem_loaded(o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                        tmem_st32(tO + c * 32, o);
                    }
                    tmem_wait_st();
                }
                m = m_new;
            }
            // (a row without a score above -inf so far: the first one there is goes beyond any threshold, so that it becomes the reference)
            const float neg_m = m == -INFINITY ? kNoReference : kWeightShift - m;
            const uint64_t neg_m_x2 = pack_f32x2(neg_m, neg_m), scale2_x2 = pack_f32x2(scale2, scale2);
            uint64_t ex_a = 0ull, ex_b = 0ull;
            uint32_t buf[2][32];
            tmem_ld32(tMine, buf[0]);
            tmem_ld32(tMine + 32, buf[1]);
            tmem_wait_ld();
            tmem_loaded(buf[0]);
            tmem_loaded(buf[1]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float k0 = kscale[2 * c], k1 = kscale[2 * c + 1];
                const uint64_t k0_x2 = pack_f32x2(k0, k0), k1_x2 = pack_f32x2(k1, k1);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float x0, x1;
                    const uint64_t product = mul_f32x2(pack_f32x2(__uint_as_float(buf[c][2 * j]), __uint_as_float(buf[c][2 * j + 1])), scale2_x2);
                    const uint64_t xx = fma_f32x2(product, j < 8 ? k0_x2 : k1_x2, neg_m_x2);
                    unpack_f32x2(xx, x0, x1);
                    const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
                    pk[c * 16 + j] = pack2_16bit<true>(p0, p1);
                    const uint64_t pe = pack_f32x2(p0, p1);
                    if (j & 1) ex_b = add_f32x2(ex_b, pe);
                    else ex_a = add_f32x2(ex_a, pe);
                }
            }
            float b0, b1;
            unpack_f32x2(add_f32x2(ex_a, ex_b), b0, b1);
            sum = b0 + b1;
            // No weight can exceed the sum: one of at most 2^(8 + 7) means that no score is more than 2^8 above its reference.  All
            // threads have read S when they meet here: P, which lies in S's first columns, may be stored.
            if (!any_of(7, both, sum > kWeightLimit) || tries == 2) break;
        }
        tmem_st32(tS + 32 * s, pk);
        l += sum;
        tmem_wait_st();
        tc_fence_before();
        asm volatile("bar.arrive %0, %1;" ::"r"(9 + p_bar), "r"(both + 32) : "memory");      // hand-off of P, once per tile on every path
        if (++b == 3u) b = 0;
        if (++p_bar == 3u) p_bar = 0;
    }
    // an idle warp has seen none of the phases: they are what the others' are
    if (idle)
        for (int i = 0; i < T; ++i) { phases ^= 1u << b; if (++b == 3u) b = 0; }
    // ---- segment end
    k->sum[s][wtid] = l;
    if (!idle) mbar_wait_certain(smem_u32(&aux->joint_o_done), done_phase & 1u, &aux->abort_flag);
    tc_fence_after();
    meet_at_segment_end(aux, js);          // both warpgroups done: all MMAs of the segment have completed
    const volatile Segment& again = aux->seg[js.seg_no % kSegs];
    const bool bad = const_cast<volatile int&>(aux->seg_bad_tree) || again.bad_page;
    const bool write_ok = !bad && !*const_cast<volatile int*>(&aux->abort_flag);
    const long long part_base = (2ll * blockIdx.x + (js.seg_no > 0 ? 1 : 0)) * kPartialRows;
    const int node = (int)row_node(p, rr);
    const long long out_row = rr < again.M ? (long long)(again.node_base + node) * p.num_q_heads + again.h * G + (rr - node * G) : 0;
    const bool row_ok = write_ok && rr < again.M, whole = again.tile0 == 0 && again.tile1 == again.tiles;
    // staging for coalesced stores: Q is idle now
    float* stage = reinterpret_cast<float*>(smem + (s * 4 + ((threadIdx.x >> 5) & 3)) * kStageBytesPerWarp);
    const float lt = k->sum[0][wtid] + k->sum[1][wtid], w = lt > 0.f ? 1.f / lt : 0.f;
    tc_fence_after();
#pragma unroll 1
    for (int c4 = 2 * s; c4 < (idle ? 0 : 2 * s + 2); ++c4) {
        uint32_t o[32];
        tmem_ld32(tmem + lane_sel + kJointO + c4 * 32, o);
        tmem_wait_ld();
        tmem_loaded(o);
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(o[j]) * w;
        if (whole) store_rows32<kF16>(p, stage, out_row, row_ok, c4 * 32, v);
        else if (row_ok) {
            // a partial: [32 groups of four channels][rows][4]
            float4* part = reinterpret_cast<float4*>(p.part_o) + part_base * 32 + rr;
#pragma unroll
            for (int j = 0; j < 8; ++j) part[(c4 * 8 + j) * kPartialRows] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
    }
    if (s == 0 && rr < again.M) {
        const float lse = lse_of_sum(m, lt);
        if (!write_ok) {
            if (bad && !whole) p.part_lse[part_base + rr] = __uint_as_float(kBadPartial);      // the merge leaves the row alone
        } else if (!whole) p.part_lse[part_base + rr] = lse;
        else if (p.lse) p.lse[out_row] = lse;
    }
}

// ------------------------------------------------------------------------------------------ joint units, keys on lanes
// Thread = key of the tile, in both warpgroups; warpgroup s has kHalf of the unit's rows, from row s * kHalf on.  A row's numbers (scale,
// reference) lie in shared memory and are the same for the warpgroup's four warps, which agree after each tile on whether all
// scores stayed within the lazy threshold of their rows' references.  `sum`: the weights of pairs of rows over this thread's keys.
template <int kHalf, bool kF16>
struct KeysStream {
    const AttnParams& p;
    AuxFp8* aux;
    KeysScratch* k;
    uint32_t tmem, tS;               // tS: of the tile, this warp's lanes and this warpgroup's rows
    unsigned char* p_row;            // this key's row of the tile's P, from this warpgroup's rows on
    int s, wtid;
    uint64_t sum[kHalf / 2];

    static constexpr int kRows = 2 * kHalf;
    __device__ __forceinline__ int row0() const { return s * kHalf; }
    __device__ __forceinline__ void begin(const Segment& g) {
        if (wtid < kHalf) {
            const int row = row0() + wtid;
            // rows beyond M: weights of 0; others: any score at all is above the threshold until the first reference is there
            k->scale[row] = row < g.M ? score_scale(p, aux->row_scale[row]) : 0.f;
            k->bias[row] = row < g.M ? kNoReference : -INFINITY;
            k->m[row] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < kHalf / 2; ++r) sum[r] = 0ull;
        named_barrier(7 + s, 128);
    }
    // scores of 16 rows from the warpgroup's row `r0` on, without their scales: the pieces' columns added up
    struct Columns { uint32_t a[kPieces<kF16>][16]; };
    __device__ __forceinline__ void ask(int r0, Columns& c) {
#pragma unroll
        for (int piece = 0; piece < kPieces<kF16>; ++piece) tmem_ld16(tS + piece * kRows + r0, c.a[piece]);
    }
    __device__ __forceinline__ void add_up(Columns& c, uint64_t (&x)[8]) {
#pragma unroll
        for (int piece = 0; piece < kPieces<kF16>; ++piece) {
            tmem_loaded(c.a[piece]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint64_t y = pack_f32x2(__uint_as_float(c.a[piece][2 * j]), __uint_as_float(c.a[piece][2 * j + 1]));
                x[j] = piece == 0 ? y : add_f32x2(x[j], y);
            }
        }
    }
    // The tile reaches drafted positions (or the end of the sequence): what a row does not see gets a score of -inf, in tensor memory.  A slot
    // past the end may have held a NaN, so all its pieces are replaced.
    __device__ __forceinline__ void mask(const Segment& g, int t) {
        const int j = t * kTileKeys + wtid - g.L;              // this key as a drafted node; below 0: context
#pragma unroll 1
        for (int r0 = 0; r0 < kHalf; r0 += 16) {
            uint32_t sees = 0u;
#pragma unroll 1
            for (int r = 0; r < 16; ++r) {
                const int row = row0() + r0 + r;
                const bool yes = j < 0 || (row < g.M && j < kMaxNodes && (aux->anc[row_node(p, row)] >> j & 1ull));
                sees |= yes ? 1u << r : 0u;
            }
#pragma unroll 1
            for (int piece = 0; piece < kPieces<kF16>; ++piece) {
                uint32_t a[16];
                tmem_ld16(tS + piece * kRows + r0, a);
                tmem_wait_ld();
                tmem_loaded(a);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(sees >> r & 1u)) a[r] = piece == 0 ? 0xff800000u : 0u;
                tmem_st16(tS + piece * kRows + r0, a);
            }
        }
        tmem_wait_st();
    }
    // Weights against the rows' references, to P and into `sum`; true if some score is above its reference by more than the
    // threshold.  Weights stop at 2^15.5 (a NaN stays one), so that in that case they can be taken out of `sum` again (kBack; P is
    // then written anew): what that leaves in it is 2^-24 of a sum that the new reference makes small.
    template <bool kBack>
    __device__ __forceinline__ bool weigh(float kscale) {
        const uint64_t ks_x2 = pack_f32x2(kscale, kscale);
        __half2 top = __float2half2_rn(0.f);
        Columns col[kHalf / 16];
#pragma unroll
        for (int h = 0; h < kHalf / 16; ++h) ask(16 * h, col[h]);
        tmem_wait_ld();
#pragma unroll
        for (int h = 0; h < kHalf / 16; ++h) {
            uint64_t x[8];
            uint32_t pk[8];
            add_up(col[h], x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const ulonglong2 sc = *reinterpret_cast<const ulonglong2*>(&k->scale[row0() + 16 * h + 4 * j]);
                const ulonglong2 bi = *reinterpret_cast<const ulonglong2*>(&k->bias[row0() + 16 * h + 4 * j]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint64_t y = fma_f32x2(mul_f32x2(x[2 * j + i], i ? sc.y : sc.x), ks_x2, i ? bi.y : bi.x);
                    float y0, y1;
                    unpack_f32x2(y, y0, y1);
                    const float p0 = fast_exp2(min_or_nan(y0, 15.5f)), p1 = fast_exp2(min_or_nan(y1, 15.5f));
                    pk[2 * j + i] = pack2_16bit<true>(p0, p1);
                    top = __hmax2(top, *reinterpret_cast<const __half2*>(&pk[2 * j + i]));
                    uint64_t& to = sum[8 * h + 2 * j + i];
                    to = add_f32x2(to, kBack ? pack_f32x2(-p0, -p1) : pack_f32x2(p0, p1));
                }
            }
            if constexpr (!kBack) {
                // P: keys' rows of 128 bytes, 16-byte piece c at place c ^ (key & 7); MN-major operand
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    *reinterpret_cast<uint4*>(p_row + (((row0() / 8 + 2 * h + c) ^ (wtid & 7)) << 4)) = make_uint4(pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
            }
        }
        return __low2float(top) > kWeightLimit || __high2float(top) > kWeightLimit;
    }
    // The rows' references move up to the tile's largest scores.
    __device__ __forceinline__ void raise(float kscale, bool first, uint32_t seq) {
        const int lane = wtid & 31, warp = wtid >> 5;
        unsigned most = 0u;                                    // lane i's: of the warpgroup's row i over the warp's keys
#pragma unroll 1
        for (int h = 0; h < kHalf; h += 16) {
            uint64_t x[8];
            Columns col;
            ask(h, col);
            tmem_wait_ld();
            add_up(col, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y[2];
                unpack_f32x2(x[j], y[0], y[1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const unsigned u = __reduce_max_sync(0xffffffffu, ordered(y[i] * k->scale[row0() + h + 2 * j + i] * kscale));
                    if (lane == h + 2 * j + i) most = u;
                }
            }
        }
        if (lane < kHalf) k->most[warp][row0() + lane] = most;
        named_barrier(7 + s, 128);
        bool moved = false;
        if (wtid < kHalf) {
            const int row = row0() + wtid;
            const float m = k->m[row];
            const float m_new = fmaxf(m, from_ordered(max(max(k->most[0][row], k->most[1][row]), max(k->most[2][row], k->most[3][row]))));
            moved = k->bias[row] > -INFINITY && m_new > m;
            k->alpha[row] = moved ? fast_exp2(m - m_new) : 1.f;
            if (moved) { k->m[row] = m_new; k->bias[row] = kWeightShift - m_new; }
        }
        if (!any_of(7 + s, 128, moved) || first) return;       // (nothing has been added up yet)
#pragma unroll
        for (int r = 0; r < kHalf / 2; ++r) sum[r] = mul_f32x2(sum[r], pack_f32x2(k->alpha[row0() + 2 * r], k->alpha[row0() + 2 * r + 1]));
        wait_for_product(aux, seq - 1u);
        const uint32_t tO = tmem + kJointO + row0();
#pragma unroll 1
        for (int h = 0; h < kHalf; h += 16) {
            uint32_t o[16];
            tmem_ld16(tO + h, o);
            tmem_wait_ld();
            tmem_loaded(o);
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * k->alpha[row0() + h + r]);
            tmem_st16(tO + h, o);
        }
        tmem_wait_st();
    }
    __device__ __forceinline__ void tile(float kscale, bool first, uint32_t seq) {
        if (!first) {
            if (!any_of(7 + s, 128, weigh<false>(kscale))) return;
            weigh<true>(kscale);
        }
        raise(kscale, first, seq);
        weigh<false>(kscale);
    }
    // the sums over the keys: lane i of each warp leaves row i's over the warp
    __device__ __forceinline__ void finish() {
        const int lane = wtid & 31, warp = wtid >> 5;
        float v[kHalf];
#pragma unroll
        for (int i = 0; i < kHalf / 2; ++i) unpack_f32x2(sum[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int o = kHalf / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < o; ++i) {
                const bool up = lane & o;
                const float send = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
            }
        if (kHalf == 16) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
        if (lane < kHalf) k->sum[warp][row0() + lane] = v[0];
    }
};

template <int kHalf, bool kWide, bool kF16>
__device__ __forceinline__ void keys_segment(const AttnParams& p, AuxFp8* aux, unsigned char* smem, uint32_t tmem, const int s, const JointSegment& js,
                                             uint32_t& phases, const uint32_t done_phase) {
    constexpr int kRows = 2 * kHalf;
    constexpr uint32_t kColumns = kPieces<kF16> * kRows;
    const Segment& g = js.g;
    const int wtid = threadIdx.x - 128 - s * 128;
    const uint32_t lane_sel = (uint32_t)(((threadIdx.x >> 5) & 3) * 32) << 16;
    KeysScratch* k = reinterpret_cast<KeysScratch*>(smem + kScratchOff<kWide, kF16>);
    const int T = g.tile1 - g.tile0;
    {
        KeysStream<kHalf, kF16> ks{p, aux, k, tmem + lane_sel, 0u, nullptr, s, wtid, {}};
        ks.begin(g);
        uint32_t b = 0, p_bar = 0;
        for (int i = 0; i < T; ++i) {
            const int t = g.tile0 + i;
            const uint32_t seq = js.tile_base + (uint32_t)i;
            wait_for_scores(aux, b, phases);
            if (i >= 2) wait_for_product(aux, seq - 2u);           // the last reader of this P
            ks.tS = tmem + lane_sel + joint_s(b, kColumns) + s * kHalf;
            ks.p_row = smem + kPOff<kF16> + (i & 1) * kPBytes + wtid * 128;
            if ((t + 1) * kTileKeys > g.L) ks.mask(g, t);
            ks.tile(aux->note[seq % kNotes].kscale[wtid >> 4], i == 0, seq);
            fence_proxy_async_smem();                  // P is read by the product
            tc_fence_before();
            asm volatile("bar.arrive %0, 288;" ::"r"(9 + p_bar) : "memory");      // hand-off of P, once per tile on every path
            if (++b == joint_buffers(kColumns)) b = 0;
            if (++p_bar == 3u) p_bar = 0;
        }
        ks.finish();
    }
    mbar_wait_certain(smem_u32(&aux->joint_o_done), done_phase & 1u, &aux->abort_flag);
    tc_fence_after();
    meet_at_segment_end(aux, js);          // both warpgroups done: all MMAs of the segment have completed
    const volatile Segment& again = aux->seg[js.seg_no % kSegs];
    const bool bad = const_cast<volatile int&>(aux->seg_bad_tree) || again.bad_page;
    const bool write_ok = !bad && !*const_cast<volatile int*>(&aux->abort_flag);
    const long long part_base = (2ll * blockIdx.x + (js.seg_no > 0 ? 1 : 0)) * kPartialRows;
    const int M = again.M, node_base = again.node_base, h = again.h, G = p.group;
    const bool whole = again.tile0 == 0 && again.tile1 == again.tiles;
    tc_fence_after();
    auto out_row_of = [&](int row) {
        const int node = (int)row_node(p, row);
        return (long long)(node_base + node) * p.num_q_heads + h * G + (row - node * G);
    };
    if (wtid < kHalf) {
        const int row = s * kHalf + wtid;
        const float l = (k->sum[0][row] + k->sum[1][row]) + (k->sum[2][row] + k->sum[3][row]);
        k->w[row] = l > 0.f ? 1.f / l : 0.f;
        if (row < M) {
            if (write_ok) {
                const float lse = lse_of_sum(k->m[row], l);
                if (!whole) p.part_lse[part_base + row] = lse;
                else if (p.lse) p.lse[out_row_of(row)] = lse;
            } else if (bad && !whole) {
                p.part_lse[part_base + row] = __uint_as_float(kBadPartial);      // the merge leaves the row alone
            }
        }
    }
    named_barrier(7 + s, 128);
    // Lane = channel: a warp's 32 channels of a row are neighbours.
#pragma unroll 1
    for (int r0 = s * kHalf; r0 < s * kHalf + kHalf; r0 += 16) {
        uint32_t o[16];
        tmem_ld16(tmem + lane_sel + kJointO + r0, o);
        // the next head's row, after a node's last head the next node's first (few instructions: they are fetched cold)
        uint16_t* out = reinterpret_cast<uint16_t*>(p.out) + out_row_of(r0) * kHeadDim + wtid;
        const long long wrap = (long long)(p.num_q_heads - G) * kHeadDim;
        int hg = r0 - (int)row_node(p, r0) * G;
        float* part = p.part_o + (part_base * 32 + (long long)(wtid >> 2) * kPartialRows + r0) * 4 + (wtid & 3);
        const int rows = write_ok ? M - r0 : 0;
        tmem_wait_ld();
        tmem_loaded(o);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float v = __uint_as_float(o[r]) * k->w[r0 + r];
            if (r < rows) {
                if (whole) *out = (uint16_t)pack2_16bit<kF16>(v, 0.f);
                else part[4 * r] = v;
            }
            out += kHeadDim;
            if (++hg == G) { hg = 0; out += wrap; }
        }
    }
}

// ------------------------------------------------------------------------------------------ shared units
// The weights of a tile against the running maximum m, 32 columns of S at a time.  False, with nothing stored, if some
// row's weights show that a score may exceed m by more than the lazy threshold (`force`: this row's do).
__device__ __forceinline__ bool weigh_tile(const uint32_t tS, const float* kscale, const float scale2, const float m, float& l, bool& force) {
    const uint64_t neg_m_x2 = pack_f32x2(kWeightShift - m, kWeightShift - m);
    uint64_t ex_a = 0ull, ex_b = 0ull;
    uint32_t pk[64];
    uint32_t buf_a[32], buf_b[32];
    tmem_ld32(tS, buf_a);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t (&cur)[32] = (c & 1) ? buf_b : buf_a;
        uint32_t (&nxt)[32] = (c & 1) ? buf_a : buf_b;
        const float s0 = kscale[2 * c] * scale2, s1 = kscale[2 * c + 1] * scale2;
        const uint64_t s0_x2 = pack_f32x2(s0, s0), s1_x2 = pack_f32x2(s1, s1);
        tmem_wait_ld();
        tmem_loaded(cur);
        if (c < 3) tmem_ld32(tS + (c + 1) * 32, nxt);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float x0, x1;
            const uint64_t xx = fma_f32x2(pack_f32x2(__uint_as_float(cur[2 * j]), __uint_as_float(cur[2 * j + 1])), j < 8 ? s0_x2 : s1_x2, neg_m_x2);
            unpack_f32x2(xx, x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            pk[c * 16 + j] = pack2_16bit<true>(p0, p1);
            const uint64_t pe = pack_f32x2(p0, p1);
            if (j & 1) ex_b = add_f32x2(ex_b, pe);
            else ex_a = add_f32x2(ex_a, pe);
        }
    }
    float b0, b1;
    unpack_f32x2(add_f32x2(ex_a, ex_b), b0, b1);
    force = (b0 + b1) > kWeightLimit;
    if (__any_sync(0xffffffffu, force)) return false;
    tmem_st32(tS, reinterpret_cast<uint32_t(&)[32]>(pk[0]));
    tmem_st32(tS + 32, reinterpret_cast<uint32_t(&)[32]>(pk[32]));
    l += b0 + b1;
    return true;
}

// Stream s has rows [128 s, 128 s + 128); `it`: S tiles of the CTA's earlier shared segments.
template <bool kF16>
__device__ __forceinline__ void shared_segment(const AttnParams& p, AuxFp8* aux, unsigned char* smem, uint32_t tmem, const int s, const JointSegment& js,
                                               const uint32_t it, const uint32_t od_phase) {
    constexpr uint32_t kPlaces = kRawTiles<true, kF16>;
    const Segment& g = js.g;
    const int wtid = threadIdx.x - 128 - s * 128, G = p.group;
    volatile int* abort_flag = &aux->abort_flag;
    const uint32_t lane_sel = (uint32_t)(((threadIdx.x >> 5) & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_sel + s * 128, tO = tS + 256;
    const int rr = s * 128 + wtid, T = g.tile1 - g.tile0;
    const unsigned long long anc_row = rr < g.M ? aux->anc[row_node(p, rr)] : 0ull;
    const float scale2 = score_scale(p, aux->row_scale[rr]);
    float m = -INFINITY, l = 0.f;
    bool near = false;                   // all of the warp's rows have a reference, and none a far one
    for (int i = 0; i < T; ++i) {
        const int t = g.tile0 + i;
        const uint32_t seq = js.tile_base + (uint32_t)i;
        mbar_wait_certain(smem_u32(&aux->s_full[s]), (it + i) & 1u, abort_flag);
        tc_fence_after();
        const float* kscale = aux->note[seq % kNotes].kscale;
        if ((t + 1) * kTileKeys > g.L) {
            // the mask of the drafted positions (rows_segment), over 128 keys
            const int j0 = t * kTileKeys - g.L;
            unsigned long long lo, hi;
            if (j0 >= 0) {
                lo = j0 < 64 ? anc_row >> j0 : 0ull;
                hi = 0ull;
            } else {
                const int k = -j0;   // 1..127 prefix keys at the front of the tile
                if (k >= 64) { lo = ~0ull; hi = (k == 64 ? 0ull : (~0ull >> (128 - k))) | (anc_row << (k - 64)); }
                else { lo = (~0ull >> (64 - k)) | (anc_row << k); hi = anc_row >> (64 - k); }
            }
#pragma unroll 1
            for (int c4 = 0; c4 < 4; ++c4) {
                const uint32_t bits = (uint32_t)((c4 < 2 ? lo : hi) >> ((c4 & 1) * 32));
                uint32_t r[32];
                tmem_ld32(tS + c4 * 32, r);
                tmem_wait_ld();
                tmem_loaded(r);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (!((bits >> j) & 1u)) r[j] = 0xff800000u;   // -inf
                tmem_st32(tS + c4 * 32, r);
            }
            tmem_wait_st();
        }
        bool done = false, force = false;
        if (near) done = weigh_tile(tS, kscale, scale2, m, l, force);
        if (!done) {
            // The long way: the tile's maximum first, then the weights; twice over tensor memory and rolled, because
            // it runs on a segment's first tile, after a jump of the maximum and on rows of no or a far reference only.
            float mx = -INFINITY;
#pragma unroll 1
            for (int c4 = 0; c4 < 4; ++c4) {
                uint32_t r[32];
                tmem_ld32(tS + c4 * 32, r);
                tmem_wait_ld();
                tmem_loaded(r);
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    float a = __uint_as_float(r[16 * hf]);
#pragma unroll
                    for (int j = 1; j < 16; ++j) a = fmaxf(a, __uint_as_float(r[16 * hf + j]));
                    mx = fmaxf(mx, a * (kscale[2 * c4 + hf] * scale2));
                }
            }
            const float m_new = fmaxf(m, mx);
            // (false when both are -inf: NaN compares false)  A tile sent here by the fast path's sum moves m up at once.
            const bool need = force ? m_new > m : (m_new - m) > kLazyRescale;
            if (__any_sync(0xffffffffu, need)) {
                const float alpha = (m_new == -INFINITY) ? 1.f : fast_exp2(m - m_new);
                if (i > 0) {
                    // S of this tile is here, and its product was issued after O += P V of the tile before: the
                    // commit that announced S covers that product too, so O may be touched now
                    tc_fence_after();
#pragma unroll 1
                    for (int c4 = 0; c4 < 4; ++c4) {
                        uint32_t o[32];
                        tmem_ld32(tO + c4 * 32, o);
                        tmem_wait_ld();
                        tmem_loaded(o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                        tmem_st32(tO + c4 * 32, o);
                    }
                    tmem_wait_st();
                    l *= alpha;
                }
                m = m_new;
            }
            near = !__any_sync(0xffffffffu, fabsf(m) >= kFarReference);
            const float neg_m = (m == -INFINITY) ? 0.f : kWeightShift - m;
            float sum = 0.f;
#pragma unroll 1
            for (int c4 = 0; c4 < 4; ++c4) {
                // the weights of 32 keys take columns that hold only scores already read (16 c4 + 16 <= 32 (c4 + 1))
                uint32_t sv[32], pk[16];
                tmem_ld32(tS + c4 * 32, sv);
                tmem_wait_ld();
                tmem_loaded(sv);
                float x_a = 0.f, x_b = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float sc = kscale[2 * c4 + (j >> 3)] * scale2;
                    const float p0 = fast_exp2(__fadd_rn(__fmul_rn(__uint_as_float(sv[2 * j]), sc), neg_m));
                    const float p1 = fast_exp2(__fadd_rn(__fmul_rn(__uint_as_float(sv[2 * j + 1]), sc), neg_m));
                    pk[j] = pack2_16bit<true>(p0, p1);
                    x_a += p0; x_b += p1;
                }
                tmem_st16(tS + c4 * 16, pk);
                sum += x_a + x_b;
            }
            l += sum;
        }
        tmem_wait_st();
        tc_fence_before();
        // V of the tile has been turned into fp16 (stream 1's product follows stream 0's).  A wait that gives up raises the abort flag; the
        // arrivals happen all the same.
        if (s == 0 && wtid < 32) {
            mbar_wait(smem_u32(&aux->v_full[seq % kFp8VSlots]), (seq / kFp8VSlots) & 1u, abort_flag);
            __syncwarp();
        }
        // Hand-off of P on hardware barrier 4 + s, once per key tile of this stream, on every path (softmax_loop)
        asm volatile("bar.arrive %0, 160;" ::"r"(4 + s) : "memory");
        // the next K tile has landed (hardware barrier 6, T - 1 times; softmax_loop)
        if (s == 0 && wtid < 32 && i + 1 < T) {
            mbar_wait(smem_u32(&aux->raw_full[2u * ((seq + 1u) % kPlaces)]), ((seq + 1u) / kPlaces) & 1u, abort_flag);
            __syncwarp();
            asm volatile("bar.arrive 6, 64;" ::: "memory");
        }
    }
    // ---- segment end: every product of this stream has completed
    mbar_wait_certain(smem_u32(&aux->o_done[s]), od_phase & 1u, abort_flag);
    tc_fence_after();
    meet_at_segment_end(aux, js);          // both streams done: all MMAs of the segment have completed
    const volatile Segment& again = aux->seg[js.seg_no % kSegs];
    const bool bad = const_cast<volatile int&>(aux->seg_bad_tree) || again.bad_page;
    const bool write_ok = !bad && !*abort_flag;
    const long long part_base = (2ll * blockIdx.x + (js.seg_no > 0 ? 1 : 0)) * kPartialRows;
    const int node = (int)row_node(p, rr);
    const long long out_row = rr < again.M ? (long long)(again.node_base + node) * p.num_q_heads + again.h * G + (rr - node * G) : 0;
    const bool row_ok = write_ok && rr < again.M, whole = again.tile0 == 0 && again.tile1 == again.tiles;
    float* stage = reinterpret_cast<float*>(smem + (s * 4 + ((threadIdx.x >> 5) & 3)) * kStageBytesPerWarp);
    const float w = l > 0.f ? 1.f / l : 0.f;
    tc_fence_after();
#pragma unroll 1
    for (int c4 = 0; c4 < 4; ++c4) {
        uint32_t o[32];
        tmem_ld32(tO + c4 * 32, o);
        tmem_wait_ld();
        tmem_loaded(o);
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(o[j]) * w;
        if (whole) store_rows32<kF16>(p, stage, out_row, row_ok, c4 * 32, v);
        else if (row_ok) {
            float4* part = reinterpret_cast<float4*>(p.part_o) + part_base * 32 + rr;
#pragma unroll
            for (int j = 0; j < 8; ++j) part[(c4 * 8 + j) * kPartialRows] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
    }
    if (rr < again.M) {
        const float lse = lse_of_sum(m, l);
        if (!write_ok) {
            if (bad && !whole) p.part_lse[part_base + rr] = __uint_as_float(kBadPartial);
        } else if (!whole) p.part_lse[part_base + rr] = lse;
        else if (p.lse) p.lse[out_row] = lse;
    }
}

// The segment's results are stored: those of rows that see a drafted node whose V has a NaN become one, channel by channel, from the
// rows of V in the cache (convert_loop left the NaNs out; a thread per row of the unit).
__device__ __forceinline__ void mark_nan_drafts(const AttnParams& p, AuxFp8* aux, uint32_t seg_no) {
    const volatile Segment& g = aux->seg[seg_no % kSegs];
    const int row = threadIdx.x - 128, L = g.L, G = p.group;
    if (row >= g.M || const_cast<volatile int&>(aux->seg_bad_tree) || g.bad_page || *const_cast<volatile int*>(&aux->abort_flag)) return;
    const int node = (int)row_node(p, row);
    const long long out_row = (long long)(g.node_base + node) * p.num_q_heads + g.h * G + (row - node * G);
    float* part = p.part_o + ((2ll * blockIdx.x + (seg_no > 0 ? 1 : 0)) * kPartialRows * 32 + row) * 4;      // [32 groups of four channels][rows][4]
    const bool whole = g.tile0 == 0 && g.tile1 == g.tiles;
#pragma unroll 1
    for (unsigned long long seen = aux->anc[node]; seen; seen &= seen - 1ull) {
        const int pos = L + __ffsll((long long)seen) - 1;
        const int page = p.block_table[(long long)g.b * p.max_pages_per_seq + (pos >> p.page_shift)];
        const uint8_t* v = reinterpret_cast<const uint8_t*>(p.v_cache) +
                           (((long long)page * p.num_kv_heads + g.h) * p.page_size + (pos & (p.page_size - 1))) * kHeadDim;
#pragma unroll 1
        for (int c = 0; c < kHeadDim; ++c) {
            if ((unsigned)page >= (unsigned)p.num_pages || (v[c] & 0x7f) != 0x7f) continue;
            if (whole) reinterpret_cast<uint16_t*>(p.out)[out_row * kHeadDim + c] = 0x7fff;      // a NaN of either type
            else part[(c >> 2) * (kPartialRows * 4) + (c & 3)] = __int_as_float(0x7fffffff);
        }
    }
}

// ------------------------------------------------------------------------------------------ softmax warpgroups
template <bool kWide, bool kF16>
__device__ __forceinline__ void softmax_loop_fp8(const AttnParams& p, AuxFp8* aux, unsigned char* smem, uint32_t tmem, const int s /*warpgroup*/) {
    const int wtid = threadIdx.x - 128 - s * 128;          // 0..127 inside the warpgroup; TMEM lane
    uint32_t seg_no = 0, tile_base = 0;          // segments and key tiles so far
    uint32_t phases = 0, joint_segs = 0;         // joint units: phases of the S buffers' barriers, segments
    uint32_t shared_it = 0, shared_segs = 0;     // shared units: tiles, segments
    const bool leader = s == 0 && wtid < 32;
    meet_before_segment(aux, 0, leader);
    for (;;) {
        const Segment g = announced_segment(aux, seg_no);
        if (g.tile1 == 0) break;
        const int keys = keys_rows(g.M);         // keys on lanes: the padded rows
        int parent_i = -1;
        if (s == 0 && wtid < g.n) parent_i = p.tree_parent[g.node_base + wtid];
        if (seg_no > 0) named_barrier(1, 256);   // the other warpgroup may still be reading its staging area in the Q block
        if (leader) const_cast<volatile int&>(aux->seg_reached) = (int)seg_no;
        {
            // shared: a block of 128 rows for each warpgroup; else each loads half of the rows
            const int half = keys ? keys >> 1 : 64, r_in_8 = wtid >> 4;
            const int first = g.shared ? r_in_8 : half * s + r_in_8;
            load_q_fp8<kF16>(p, g, aux, smem + (g.shared ? s * kPieces<kF16> * kPieceBytes : 0) + first * 128, keys ? keys * 128 : kPieceBytes,
                             (g.shared ? 128 * s : 0) + first, g.shared ? 16 : half >> 3, wtid & 15);
        }
        if (s == 0) {
            if (wtid == 0) aux->seg_bad_tree = 0;
            named_barrier(2, 128);
            if (wtid < g.n) {
                const bool bad = (wtid == 0 && parent_i != -1) || (wtid > 0 && (parent_i < 0 || parent_i >= wtid));
                if (bad) {
                    atomicExch(&aux->seg_bad_tree, 1);
                    report(p.status, kErrBadTree);
                }
                aux->parent[wtid] = bad ? (short)-1 : (short)parent_i;
            }
            named_barrier(2, 128);
            if (wtid < g.n) {
                unsigned long long m = 0;
                if (!aux->seg_bad_tree)
                    for (int j = wtid, guard = 0; j >= 0 && guard < kMaxNodes; j = aux->parent[j], ++guard) m |= 1ull << j;
                aux->anc[wtid] = m;
            }
        }
        fence_proxy_async_smem();
        named_barrier(1, 256);                 // masks and the tree verdict are visible to both warpgroups
        mbar_arrive(smem_u32(&aux->q_full));

        const JointSegment js{g, tile_base, seg_no, leader};
        if (kWide && g.shared) {
            shared_segment<kF16>(p, aux, smem, tmem, s, js, shared_it, shared_segs);
            shared_it += (uint32_t)(g.tile1 - g.tile0);
            ++shared_segs;
        } else {
            if (keys == 32) keys_segment<16, kWide, kF16>(p, aux, smem, tmem, s, js, phases, joint_segs);
            else if (keys) keys_segment<32, kWide, kF16>(p, aux, smem, tmem, s, js, phases, joint_segs);
            else rows_segment<kWide, kF16>(p, aux, smem, tmem, s, js, phases, joint_segs);
            ++joint_segs;
        }
        tc_fence_before();
        tile_base += (uint32_t)(g.tile1 - g.tile0);
        if (const_cast<volatile int&>(aux->mark_drafts)) {      // alike in all threads; written again only after barrier 1 of the next segment
            named_barrier(1, 256);               // the results, which other threads have stored
            mark_nan_drafts(p, aux, seg_no);
        }
        ++seg_no;
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
        for (int i = 0; i < kRawTiles<kWide, kF16>; ++i)
            for (int kv = 0; kv < 2; ++kv) {
                mbar_init(smem_u32(&aux->raw_full[2 * i + kv]), 2);            // the bytes and the note
                mbar_init(smem_u32(&aux->raw_empty[2 * i + kv]), kv ? 4 : 1);  // V: the converting warps; K: the products
            }
        for (int i = 0; i < 3; ++i) mbar_init(smem_u32(&aux->joint_s_full[i]), 1);
        mbar_init(smem_u32(&aux->joint_o_done), 1);
        for (int i = 0; i < kFp8VSlots; ++i) {
            mbar_init(smem_u32(&aux->v_full[i]), 4);
            mbar_init(smem_u32(&aux->v_empty[i]), 1);
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
            producer_loop_fp8<kWide, kF16, kManySeqs>(p, &kmap, &vmap, aux, smem_base + kRawOff<kWide, kF16>, w);
        } else if (warp == 1) {
            mma_loop_fp8<kWide, kF16>(aux, smem_base, tmem);
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (!kManySeqs) wait_for_inputs();
        convert_loop<kWide, kF16>(p, aux, smem);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        if (!kManySeqs) wait_for_inputs();
        softmax_loop_fp8<kWide, kF16>(p, aux, smem, tmem, warp >= 8 ? 1 : 0);
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
