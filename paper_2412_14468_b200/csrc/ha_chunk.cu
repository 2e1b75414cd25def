// Attention of new tokens over a paged cache: every new token (one of a decoding sequence, or a chunk of a prompt) attends to all
// cached tokens up to its own, exactly.
//
//     out_i = sum_{t <= pos_i} softmax_t(scale <q_i, k_t>) v_t,   pos_i = seq_len - n_new + i
//
// One pass over the keys with a running maximum m and sum l per row: p = 2^(s - m) in 32 bits, l += p, O += bf16(p) V; the maximum
// that the exponents refer to is raised, and O and l rescaled, only when a tile's maximum lies more than 2^8 above it, so that most
// tiles leave O alone (p <= 2^8: sums stay far inside 32 bits).  p is rounded to bf16 for the tensor cores, as V is bf16 and both
// operands have one type: at most half a step, 2^-8 relative, on each weight, of independent sign; l sums the unrounded p.
//
// Work: see ha_chunk_plan.h.  A CTA holds two tiles of 128 query rows (tokens x heads of a group, so that one fetch of K and V
// serves the whole group) and streams key tiles of 128 tokens through two rings in shared memory.
//   warps 0 - 3, 4 - 7   softmax of row tile 0 / 1: one thread per row, its 128 scores in registers
//   warp 8               issues S = Q K^T (both operands K-major, in shared memory)
//   warp 11              issues O += P V (P from tensor memory, V N-major)
//   warps 9, 10          fetch K and q / V, through the block table, into the 128-byte swizzle
// Tensor memory: O of both row tiles, P (bf16) of both, and ONE S of 128 columns that the two take turns at: scores stay there
// only until the softmax warps have them in registers, so the next S of a row tile is ready before its softmax is done with
// the last one, and neither waits for the other.  (With an S of its own for each row tile, overwritten by P, a tile's two
// products and its softmax formed one chain of 3700 cycles, 2048 of them with the tensor cores at work.)
// A unit of at most 128 rows (a decoding sequence) uses the two halves for alternate key tiles and joins them at its end.
// Fetching: by TMA, a box for the rows of one page (or 128 of them).  A box costs 45 ns and 1.3 ns a row of an issuing thread's time
// however it is issued (measured), so pages of 16 take 1.0 us for a K tile in two boxes a page (one for either half of the columns,
// which a K-major operand of 128 rows needs) and 0.85 us for a V tile in one.  By threads: the V tile that a sequence ends in, as rows behind the end have to be
// zeros (0 times what lies there need not be 0); and everything where pages have fewer than 8 tokens (the swizzle repeats every
// 8 rows) or no tensor map takes the strides.
// What bounds it: a pair of tiles (256 rows x 128 keys) is 2048 cycles of MMAs and 2048 of exponentials, and takes about 3000: a row
// tile's softmax is one chain (scores to registers 100 cycles, maximum 400, vote 110, exponentials 1400, weights and barriers 300).
// Measured: 2048 new tokens of 16384, 32 heads, pages of 16: 411 us, 1250 TFLOP/s (0.75 of a large bf16 product); 32 sequences of
// 16384 with one new token: 333 us, 6.4 TB/s; one of 4096: 17 us, a chain of latencies.
// A unit cut between CTAs: each part writes m, l and O to the workspace; the part that arrives last joins them all, in the order of
// the keys, so that results do not depend on the order of arrival.
// Every wait is bounded: a waiter that gives up raises HA_DEV_TIMEOUT and stops, those that wait for it run out as well, and the MMAs
// and copies in flight are waited for before the tensor memory is given back.
#include "ha_attn_dev.cuh"
#include "ha_chunk_plan.h"
#include "ha_encode_dev.cuh"
#include "ha_umma.cuh"

#include <cstring>
#include <type_traits>

namespace ha {

constexpr int kC_Softmax = 256;                    // threads of the softmax roles
constexpr int kC_WarpS = 8, kC_WarpK = 9, kC_WarpV = 10, kC_WarpO = 11;
constexpr int kC_Threads = 384;                    // 12 warps: 168 registers a thread
// of these, moved to the softmax warps, which hold a row of 128 scores
constexpr int kC_RegsSoftmax = 208, kC_RegsOther = 88;
static_assert(kC_RegsSoftmax * kC_Softmax + kC_RegsOther * (kC_Threads - kC_Softmax) <= 168 * kC_Threads, "no more than the block was launched with");
constexpr int kC_TileBytes = kChunkTile * kD * 2;  // 32768: two halves of 64 columns, each 128 rows of 128 bytes
constexpr int kC_Half = kC_TileBytes / 2;
constexpr int kC_SlotsK = 2, kC_SlotsV = 3;
constexpr int kC_OffQ = 0, kC_OffK = 2 * kC_TileBytes, kC_OffV = kC_OffK + kC_SlotsK * kC_TileBytes;
constexpr int kC_Smem = kC_OffV + kC_SlotsV * kC_TileBytes;   // 229376
constexpr int kC_WarpPlan = 128;                   // sequences up to which one warp finds its CTA's share
constexpr float kC_Raise = 8.0f;                   // how far (log2) a maximum may lie above the one that is referred to
constexpr uint32_t kC_ColO = 0, kC_ColS = 256, kC_ColP = 384;   // tensor-memory columns: O0, O1, S, P0, P1

struct ChunkArgs {
    const uint16_t *q;
    long long q_sn, q_sh;
    const int32_t *offsets, *seq_lens, *table;
    TensorView K, V;
    long long bt_sb;
    int n_rows, n_pages, shift, B, Hkv, log2g, causal, max_ctas, log2box;
    float scale_log2;
    uint16_t *out;
    float *lse;
    uint32_t *status;
    int32_t *tickets;
    float *part_ml, *part_acc;   // [CTA][2][256] (m, l) and [CTA][2][256][128]
};

// What a CTA does next: written by the warp that fetches keys, read by all roles.
struct ChunkPart {
    int b, h, n, row, toks, first_pos, t0, t1;       // row: of q, the unit's first; toks: 0 behind the last part
    int split, cut, first_cta, n_parts;
    int wild_v;                                      // a value that some row must not see is inf or NaN (see chunk_fetch)
};
// Part p is written when all scores of part p - 2 have been ordered.  Then row tile 0 has the scores of p - 3 and is done with p - 4, but row
// tile 1, which has nothing to do in a part of one key tile, may still be writing the results of p - 4 (it has to join in p - 3 before
// row tile 0 goes on to p - 2).  So five places are needed at least.
constexpr int kC_Parts = 8;

struct ChunkShared {
    ChunkPart parts[kC_Parts];
    unsigned long long part_full[kC_Parts];
    unsigned long long k_full[kC_SlotsK], k_empty[kC_SlotsK], v_full[kC_SlotsV], v_empty[kC_SlotsV], v_check[2], q_full, q_empty;
    unsigned long long s_full[2], s_free, p_full[2], o_done[2], joint, drained;
    long long start_rest;
    long long warp_sums[kC_Threads / 32];
    int start_b;
    int last_part;
    uint32_t tmem;
    union {
        float ml[2][128][2];     // the halves' maxima and sums, where they share a unit
        float2 joined[kChunkRows];   // of the rows of a unit whose parts are joined: maximum, one over the sum
    };
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// two 32-bit operations in one instruction
__device__ __forceinline__ void fma2(float &x, float &y, float m, float a) {   // (x, y) = (x, y) * m + a
    asm("{\n\t.reg .b64 v, f, c;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 f, {%2, %2};\n\tmov.b64 c, {%3, %3};\n\t"
        "fma.rn.f32x2 v, v, f, c;\n\tmov.b64 {%0, %1}, v;\n\t}" : "+f"(x), "+f"(y) : "f"(m), "f"(a));
}
__device__ __forceinline__ void add2(float &x, float &y, float a, float b) {
    asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %3};\n\tadd.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}"
        : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// all 128 columns of S of this thread's row
__device__ __forceinline__ void load_scores(uint32_t at, float (&v)[128]) {
    uint32_t r[4][32];
#pragma unroll
    for (int c = 0; c < 4; ++c) tmem_ld32(at + c * 32, r[c]);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 128; ++i) v[i] = __uint_as_float(r[i >> 5][i & 31]);
}

// box of a pool seen as [page][head][2 halves][slot][64]
__device__ __forceinline__ void tma_load_rows(uint32_t dst, const CUtensorMap *map, int slot, int half, int head, int page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(slot), "r"(half), "r"(head), "r"(page), "r"(bar) : "memory");
}
// box of q seen as [2 halves][row][head][64]: 128 / G tokens of G heads, half after half
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap *map, int head, int row, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(head), "r"(row), "r"(0), "r"(bar) : "memory");
}

// The fetching warps: tiles of K (and q) or of V, in the order of the parts.  log2 of the rows of a box: the rows of a V tile lie box
// by box, in either half of the columns; those of a K tile half by half.
template <bool kTma, bool kV, typename NextPart, typename Wait>
__device__ __forceinline__ void chunk_fetch(const ChunkArgs &a, NextPart next_part, const CUtensorMap *map, const CUtensorMap *map_q, ChunkShared &sh,
                                            uint32_t smem0, int lane, Wait wait) {
    ChunkPart now = {};
    constexpr int kSlots = kV ? kC_SlotsV : kC_SlotsK;
    const TensorView &T = kV ? a.V : a.K;
    unsigned long long *full = kV ? sh.v_full : sh.k_full, *empty = kV ? sh.v_empty : sh.k_empty;
    const uint32_t ring = smem0 + (kV ? kC_OffV : kC_OffK);
    const int lbox = kTma ? a.log2box : 7, lboxes = 7 - lbox;   // log2 of the rows of a box, of the boxes of a tile
    const int mask = (1 << a.shift) - 1, hw = lane >> 4, ch = lane & 15;
    int slot = 0, pending = -1;                       // pending: slot whose copies by threads are not announced yet
    uint32_t phase = 1, issued = 0, issued_q = 0;     // phase of `empty`: the ring starts empty
    bool ok = true;

    // Of a tile with tokens that some rows must not see: weight 0 times inf or NaN is not 0, so such values become 0 here, and rows that do
    // see them are given them back with the result.
    bool check = false;                               // the pending tile is one
    uint32_t part_now = 0, checks = 0, checks_issued = 0;
    bool by_tma = false;                              // ... and lands at v_check, not by this warp's own copies
    // an exponent of ones, and one more, carries into the sign's place
    auto wild_bits = [](uint32_t w) -> uint32_t { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
    auto tame = [&]() {
        const uint32_t at = ring + pending * kC_TileBytes + lane * 16;
        uint32_t any = 0;
#pragma unroll 1
        for (int i0 = 0; i0 < kC_TileBytes / 512; i0 += 16) {
            uint32_t w[16][4];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3]) : "r"(at + (i0 + i) * 512) : "memory");
#pragma unroll
            for (int i = 0; i < 16; ++i) any |= (wild_bits(w[i][0]) | wild_bits(w[i][1])) | (wild_bits(w[i][2]) | wild_bits(w[i][3]));
        }
        if (!__any_sync(0xffffffffu, any != 0)) return;
#pragma unroll 1
        for (int i = 0; i < kC_TileBytes / 128; ++i) {   // a word a lane
            const uint32_t to = ring + pending * kC_TileBytes + i * 128 + lane * 4;
            uint32_t w;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(to) : "memory");
            if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
            if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(w) : "memory");
        }
        if (lane == 0) {
            sh.parts[part_now % kC_Parts].wild_v = 1;
            __threadfence_block();
        }
    };
    // the pending tile, when all but the last kLeft groups of this warp's copies have landed
    auto announce = [&](auto left) -> bool {
        if (by_tma) {
            if (!wait(sh.v_check[checks & 1u], checks >> 1 & 1u)) return false;
            ++checks;
        } else {
            cp_async_wait<decltype(left)::value>();
        }
        __syncwarp();
        if (kV && check) tame();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&full[pending]));
        pending = -1;
        return true;
    };
    constexpr std::integral_constant<int, 0> kAll{};
    constexpr std::integral_constant<int, 1> kButOne{};
    auto bad_page = [&](int page) -> bool {           // a page outside of the pool: zeros
        if ((unsigned)page < (unsigned)a.n_pages) return false;
        if (a.status) atomicOr(a.status, HA_DEV_BAD_INDEX);
        return true;
    };
    // Page numbers for the boxes, 32 at a time, a lane each: those at work and those behind them, which are on their way
    int ahead = 0, pages0 = -1, pages1 = -1;
    auto fetch_pages = [&](int batch) {
        const int e = batch * 32 + lane;
        int page = -1;
        if ((long long)e << a.shift < now.n) {
            page = __ldcg(a.table + (long long)now.b * a.bt_sb + e);
            if (bad_page(page)) page = -1;
        }
        if (batch & 1) pages1 = page;
        else pages0 = page;
    };
    // ... and for the rows that threads copy: rows lane, lane + 32, ...
    int row_pages[4];
    auto look_up = [&](int j) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t tok = (uint32_t)j * kChunkTile + g * 32 + lane;   // a last tile may end behind 2^31
            row_pages[g] = -1;
            if (tok < (uint32_t)now.n) {
                row_pages[g] = __ldcg(a.table + (long long)now.b * a.bt_sb + (tok >> a.shift));
                if (bad_page(row_pages[g])) row_pages[g] = -1;
            }
        }
    };
    auto copy_rows = [&](int j, uint32_t dst) {       // a half-warp copies a row of 256 bytes; rows that are not there: zeros
#pragma unroll
        for (int g = 0; g < 4; ++g) {
#pragma unroll 4
            for (int i = 0; i < 16; ++i) {
                const int r = g * 32 + 2 * i + hw, page = __shfl_sync(0xffffffffu, row_pages[g], 2 * i + hw);
                const uint16_t *src = T.ptr + ch * 8;
                if (page >= 0) src += (long long)page * T.sb + (long long)now.h * T.sh + (long long)(((uint32_t)j * kChunkTile + r) & mask) * T.sn;
                const uint32_t at = kV ? ((uint32_t)(r >> lbox) << lbox) * 256 + (uint32_t)(ch >> 3) * (128u << lbox) + (uint32_t)(r & ((1 << lbox) - 1)) * 128
                                       : (uint32_t)(ch >> 3) * kC_Half + (uint32_t)r * 128;
                cp_async16(dst + at + (((ch & 7) ^ (r & 7)) << 4), src, page >= 0 ? 16u : 0u);
            }
        }
        cp_async_commit();
    };
    auto load = [&](int j, bool by_threads, bool wild) -> bool {
        if (by_threads) look_up(j);
        else {
            const int batch = (j * kChunkTile >> a.shift) >> 5;
            if (batch == ahead) fetch_pages(++ahead);
        }
        if (!mbar_test(smem_u32(&empty[slot]), phase)) {
            if (pending >= 0 && !announce(kAll)) return false;   // what is waited for may wait for it
            if (!wait(empty[slot], phase)) return false;
        }
        const uint32_t dst = ring + slot * kC_TileBytes, bar = kV && wild && !by_threads ? smem_u32(&sh.v_check[checks_issued & 1u]) : smem_u32(&full[slot]);
        if (by_threads) {
            copy_rows(j, dst);
            if (pending >= 0 && !announce(kButOne)) return false;
            pending = slot;
            check = wild;
            by_tma = false;
        } else {
            // a lane for each box; boxes behind the end of the sequence are left out (their keys are masked, whatever they are)
            const int which = lane & ((1 << lboxes) - 1), half = lane >> lboxes;
            const uint32_t tok = (uint32_t)j * kChunkTile + ((uint32_t)which << lbox);
            const int batch = (j * kChunkTile >> a.shift) >> 5;
            const int page = __shfl_sync(0xffffffffu, batch & 1 ? pages1 : pages0, (tok >> a.shift) & 31);
            const int left = now.n - j * kChunkTile, there = left >= kChunkTile ? 1 << lboxes : (left + (1 << lbox) - 1) >> lbox;
            if (lane == 0) mbar_expect_tx(bar, ((uint32_t)there << lbox) * 256);
            __syncwarp();
            if (which < there && half < (kV ? 1 : 2))
                tma_load_rows(dst + ((uint32_t)which << lbox) * (kV ? 256 : 128) + (kV ? 0 : half * kC_Half), map, tok & mask, kV ? 0 : half, now.h, page, bar);
            ++issued;
            if (kV && wild) ++checks_issued;
            if (pending >= 0 && !announce(kAll)) return false;
            if (kV && wild) {
                pending = slot;
                check = by_tma = true;
            }
        }
        __syncwarp();
        if (++slot == kSlots) { slot = 0; phase ^= 1; }
        return true;
    };
    for (uint32_t part = 0; ok && (ok = next_part(part, now)) && now.toks > 0; ++part) {
        part_now = part;
        const int t0 = now.t0, t1 = now.t1;
        const bool tail = !kTma || (kV && (long long)t1 * kChunkTile > now.n);
        // tiles from here on have tokens that the first of several new tokens must not see
        const int hidden = kV && a.causal && now.toks > 1 ? (now.first_pos + 1 > 0 ? (now.first_pos + 1) >> 7 : 0) : 0x7fffffff;
        if (kTma) {
            ahead = (t0 * kChunkTile >> a.shift) >> 5;
            fetch_pages(ahead);
        }
        for (int j = t0; ok && j < t1; ++j) {
            ok = load(j, !kTma || (tail && j == t1 - 1), j >= hidden);
            if (kV || !ok || j > t0) continue;
            // q, behind the first keys, which need not wait for its place
            if (pending >= 0 && !(ok = announce(kAll))) break;
            if (!(ok = part == 0 || wait(sh.q_empty, (part - 1) & 1u))) break;
            const int n_rows = now.toks << a.log2g, rows = n_rows <= kChunkTile ? kChunkTile : kChunkRows;
            if (kTma) {
                if (elect_one()) {
                    mbar_expect_tx(smem_u32(&sh.q_full), rows * 256);
                    for (int x = 0; x < rows / kChunkTile; ++x)
                        tma_load_q(smem0 + kC_OffQ + x * kC_TileBytes, map_q, now.h << a.log2g,
                                   now.row + x * (kChunkTile >> a.log2g), smem_u32(&sh.q_full));
                }
                ++issued_q;
            } else {
                const uint16_t *q = a.q + (long long)(now.row) * a.q_sn + (long long)(now.h << a.log2g) * a.q_sh + ch * 8;
#pragma unroll 8
                for (int r = hw; r < rows; r += 2) {
                    const bool in = r < n_rows;
                    const uint16_t *src = in ? q + (long long)(r >> a.log2g) * a.q_sn + (long long)(r & ((1 << a.log2g) - 1)) * a.q_sh : q;
                    cp_async16(smem0 + kC_OffQ + (r >> 7) * kC_TileBytes + (uint32_t)(ch >> 3) * kC_Half + (r & 127) * 128 + (((ch & 7) ^ (r & 7)) << 4), src,
                               in ? 16u : 0u);
                }
                cp_async_commit();
                cp_async_wait<0>();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.q_full));
            }
            __syncwarp();
        }
        // before the next part is waited for: what the tile shows belongs to this one
        if (ok && pending >= 0) ok = announce(kAll);
    }
    cp_async_wait<0>();
    if (!ok && kTma && kV)
        for (; checks != checks_issued; ++checks) mbar_wait_parity(smem_u32(&sh.v_check[checks & 1u]), checks >> 1 & 1u);
    if (!ok && kTma) {   // never seen: what is in flight lands (one more bounded wait each) before shared memory is given up
        for (int i = 0; i < kSlots && i < (int)issued; ++i) {
            slot = slot == 0 ? kSlots - 1 : slot - 1;
            if (slot == kSlots - 1) phase ^= 1;
            mbar_wait_parity(smem_u32(&full[slot]), phase ^ 1);
        }
        if (issued_q > 0) mbar_wait_parity(smem_u32(&sh.q_full), (issued_q - 1) & 1u);
    }
}

template <bool kTma>
__global__ void __launch_bounds__(kC_Threads, 1) chunk_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                  const __grid_constant__ CUtensorMap map_v, const ChunkArgs a) {
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ __align__(8) ChunkShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem0 = smem_u32(smem);

    if (tid == 0) {
        for (int i = 0; i < kC_Parts; ++i) mbar_init(smem_u32(&sh.part_full[i]), 1);
        for (int i = 0; i < kC_SlotsK; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 1);
            mbar_init(smem_u32(&sh.k_empty[i]), 1);
        }
        for (int i = 0; i < kC_SlotsV; ++i) {
            mbar_init(smem_u32(&sh.v_full[i]), 1);
            mbar_init(smem_u32(&sh.v_empty[i]), 1);
        }
        mbar_init(smem_u32(&sh.v_check[0]), 1);
        mbar_init(smem_u32(&sh.v_check[1]), 1);
        mbar_init(smem_u32(&sh.q_full), 1);
        mbar_init(smem_u32(&sh.q_empty), 1);
        mbar_init(smem_u32(&sh.s_free), 4);
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&sh.s_full[x]), 1);
            mbar_init(smem_u32(&sh.p_full[x]), 4);
            mbar_init(smem_u32(&sh.o_done[x]), 1);
        }
        mbar_init(smem_u32(&sh.joint), kC_Softmax / 32);
        mbar_init(smem_u32(&sh.drained), 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sh.start_b = -1;
    }
    pdl_wait();
    pdl_launch_dependents();   // nothing that a kernel reads before its own wait is written here or by anything still running
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    // ---- the whole work, and where this CTA's share of it begins: needed by the warp that walks along it, and found by that warp
    // alone (for up to kC_WarpPlan sequences) or by all of them
    auto cost_of = [&](int b, bool report) -> long long {
        if (b >= a.B) return 0;
        bool bad;
        const ChunkSeq s = chunk_seq(HA_FROM_L2(a.seq_lens + b), HA_FROM_L2(a.offsets + b), HA_FROM_L2(a.offsets + b + 1), a.n_rows, a.log2g, bad);
        if (bad && report && a.status) atomicOr(a.status, HA_DEV_BAD_INDEX);
        return a.Hkv * chunk_cost_head(s, a.log2g, a.causal);
    };
    auto ctas_for = [&](long long work) -> int { return chunk_ctas(work, a.max_ctas < (int)gridDim.x ? a.max_ctas : (int)gridDim.x); };
    // of a warp: values in front of this lane's, and all of them
    auto warp_sum = [&](long long v, long long &all) -> long long {
        long long x = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        all = __shfl_sync(0xffffffffu, x, 31);
        return x - v;
    };
    long long W = 0, rest = 0;       // rest: how far into sequence `first_b` the share begins
    int C = 1, first_b = -1;
    if (a.B <= kC_WarpPlan) {
        if (warp == kC_WarpK) {
            long long cost[kC_WarpPlan / 32], before[kC_WarpPlan / 32];
#pragma unroll
            for (int i = 0; i < kC_WarpPlan / 32; ++i) cost[i] = cost_of(i * 32 + lane, blockIdx.x == 0);
#pragma unroll
            for (int i = 0; i < kC_WarpPlan / 32; ++i) {
                long long all;
                before[i] = W + warp_sum(cost[i], all);
                W += all;
            }
            C = ctas_for(W);
            if (W > 0 && (int)blockIdx.x < C) {
                const long long f0 = chunk_bound(W, C, blockIdx.x);
#pragma unroll
                for (int i = 0; i < kC_WarpPlan / 32; ++i) {
                    const uint32_t m = __ballot_sync(0xffffffffu, before[i] <= f0 && f0 < before[i] + cost[i]);
                    if (m) {
                        const int l = __ffs(m) - 1;
                        first_b = i * 32 + l;
                        rest = f0 - __shfl_sync(0xffffffffu, before[i], l);
                    }
                }
            }
        }
    } else {
        auto block_sum = [&](long long v, long long &before) -> long long {
            long long mine;
            before = warp_sum(v, mine);
            __syncthreads();
            if (lane == 0) sh.warp_sums[warp] = mine;
            __syncthreads();
            long long all = 0;
            for (int w = 0; w < kC_Threads / 32; ++w) {
                if (w < warp) before += sh.warp_sums[w];
                all += sh.warp_sums[w];
            }
            return all;
        };
        long long before = 0;
        for (int b0 = 0; b0 < a.B; b0 += kC_Threads) W += block_sum(cost_of(b0 + tid, blockIdx.x == 0), before);
        C = ctas_for(W);
        if (W > 0 && (int)blockIdx.x < C) {
            const long long f0 = chunk_bound(W, C, blockIdx.x);
            long long done = 0;
            for (int b0 = 0; b0 < a.B; b0 += kC_Threads) {
                const long long mine = cost_of(b0 + tid, false), all = block_sum(mine, before), first = done + before;
                if (first <= f0 && f0 < first + mine) {
                    sh.start_b = b0 + tid;
                    sh.start_rest = f0 - first;
                }
                done += all;
            }
            __syncthreads();
            first_b = sh.start_b;
            rest = sh.start_rest;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    // (the answer goes by the barrier alone, so that the lanes of a warp get the same one; the roles behind one that gave up run out too)
    auto gave_up = [&]() -> bool {
        if (a.status) atomicOr(a.status, HA_DEV_TIMEOUT);
        return false;
    };
    auto wait = [&](unsigned long long &bar, uint32_t parity) -> bool {
        const uint32_t at = smem_u32(&bar);
        if (mbar_test(at, parity)) return true;
        return mbar_wait_parity(at, parity) || gave_up();
    };
    auto wait_parked = [&](unsigned long long &bar, uint32_t parity) -> bool {   // where nobody waits for the waiter
        const uint32_t at = smem_u32(&bar);
        if (mbar_test(at, parity)) return true;
        return mbar_wait_parity<0>(at, parity) || gave_up();
    };

    if (warp >= kC_WarpS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kC_RegsOther));
    {
        // the next part, by the warp that walks along the CTA's stretch, and by the others
        auto given_part = [&](uint32_t part, ChunkPart &now) -> bool {
            if (!wait(sh.part_full[part % kC_Parts], (part / kC_Parts) & 1u)) return false;
            now = sh.parts[part % kC_Parts];
            return true;
        };
        if (warp == kC_WarpK) {
            ChunkWalk walk;
            const bool busy = first_b >= 0;
            walk.W = W; walk.C = C; walk.log2g = a.log2g; walk.B = a.B; walk.Hkv = a.Hkv; walk.n_rows = a.n_rows; walk.causal = a.causal != 0;
            walk.seq_lens = a.seq_lens; walk.offsets = a.offsets;
            if (busy) walk.begin(blockIdx.x, first_b, rest);
            auto walked_part = [&](uint32_t part, ChunkPart &now) -> bool {
                now.toks = 0;
                if (busy && walk.next()) {
                    now.b = walk.b; now.h = walk.h; now.n = walk.s.n;
                    now.row = walk.s.row0 + walk.unit.tok0; now.toks = walk.unit.toks; now.first_pos = walk.unit.first_pos;
                    now.t0 = walk.t0; now.t1 = walk.t1;
                    now.split = walk.unit.split; now.cut = walk.cut; now.first_cta = walk.first_cta; now.n_parts = walk.n_parts;
                    now.wild_v = 0;
                }
                if (lane == 0) {
                    sh.parts[part % kC_Parts] = now;
                    mbar_arrive(smem_u32(&sh.part_full[part % kC_Parts]));
                }
                __syncwarp();
                return true;
            };
            chunk_fetch<kTma, false>(a, walked_part, &map_k, &map_q, sh, smem0, lane, wait_parked);
        } else if (warp == kC_WarpV) {
            chunk_fetch<kTma, true>(a, given_part, &map_v, &map_q, sh, smem0, lane, wait_parked);
        } else if (warp == kC_WarpS) {
            // ------------------------------------------------ S = Q K^T.  Item i of a part is row tile i % 2 and key tile i / 2, or, of
            // a unit of one row tile, key tile i
            constexpr uint32_t kIdesc = umma_idesc(128, 128, false);
            const uint32_t col_s = __shfl_sync(0xffffffffu, tmem, 0) + kC_ColS;
            int slot = 0;
            uint32_t phase = 0, before = 0;               // before: items so far
            bool ok = true;
            ChunkPart now = {};
            for (uint32_t part = 0; ok && (ok = given_part(part, now)) && now.toks > 0; ++part) {
                const bool split = now.split;
                const int n = (now.t1 - now.t0) * (split ? 1 : 2);
                if (!(ok = wait(sh.q_full, part & 1u))) break;
                for (int i = 0; i < n; ++i, ++before) {
                    const int x = i & 1;
                    if ((split || x == 0) && !(ok = wait(sh.k_full[slot], phase))) break;
                    if (before > 0 && !(ok = wait(sh.s_free, (before - 1) & 1u))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t qd = umma_desc_sw128(smem0 + kC_OffQ + (split ? 0 : x) * kC_TileBytes, 16, 1024);
                        const uint64_t kd = umma_desc_sw128(smem0 + kC_OffK + slot * kC_TileBytes, 16, 1024);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint64_t d = (uint64_t)((k >> 2) * (kC_Half >> 4) + (k & 3) * 2);
                            umma_ss(col_s, qd + d, kd + d, kIdesc, k ? 1u : 0u);
                        }
                        umma_commit(smem_u32(&sh.s_full[x]));
                        if (split || x == 1) umma_commit(smem_u32(&sh.k_empty[slot]));
                        if (i == n - 1) umma_commit(smem_u32(&sh.q_empty));
                    }
                    __syncwarp();
                    if ((split || x == 1) && ++slot == kC_SlotsK) { slot = 0; phase ^= 1; }
                }
            }
            // the last MMAs are complete before shared and tensor memory are given back
            if (elect_one()) umma_commit(smem_u32(&sh.drained));
            __syncwarp();
            mbar_wait_parity(smem_u32(&sh.drained), 0u);
        } else if (warp == kC_WarpO) {
            // ------------------------------------------------ O += P V, the same items
            constexpr uint32_t kIdesc = umma_idesc(128, 128, true);
            const uint32_t base = __shfl_sync(0xffffffffu, tmem, 0);
            const int lbox = kTma ? a.log2box : 7;
            // 16 tokens are two groups of 8 rows: next to one another in a box, or, of boxes of 8 rows, a box each
            const uint32_t half_bytes = 128u << lbox, group_bytes = lbox == 3 ? 2048u : 1024u;
            int slot = 0;
            uint32_t phase = 0, p_phase = 0;              // p_phase: bit x of p_full[x]
            bool ok = true;
            ChunkPart now = {};
            for (uint32_t part = 0; ok && (ok = given_part(part, now)) && now.toks > 0; ++part) {
                const bool split = now.split;
                const int n = (now.t1 - now.t0) * (split ? 1 : 2);
                for (int i = 0; i < n; ++i) {
                    const int x = i & 1;
                    if ((split || x == 0) && !(ok = wait(sh.v_full[slot], phase))) break;
                    if (!(ok = wait(sh.p_full[x], p_phase >> x & 1u))) break;
                    p_phase ^= 1u << x;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t v0 = smem0 + kC_OffV + slot * kC_TileBytes;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t r = (uint32_t)k * 16, in_box = r & ((1u << lbox) - 1);
                            const uint64_t vd = umma_desc_sw128(v0 + (r - in_box) * 256 + in_box * 128, half_bytes, group_bytes);
                            umma_ts(base + kC_ColO + x * 128, base + kC_ColP + x * 64 + k * 8, vd, kIdesc, (i >= 2 || k) ? 1u : 0u);
                        }
                        umma_commit(smem_u32(&sh.o_done[x]));
                        if (split || x == 1) umma_commit(smem_u32(&sh.v_empty[slot]));
                    }
                    __syncwarp();
                    if ((split || x == 1) && ++slot == kC_SlotsV) { slot = 0; phase ^= 1; }
                }
            }
            if (elect_one()) umma_commit(smem_u32(&sh.drained));
            __syncwarp();
            mbar_wait_parity(smem_u32(&sh.drained), 0u);
        } else {
            // ------------------------------------------------ softmax
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kC_RegsSoftmax));
            const int x = warp >> 2, row = tid & 127;
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
            const uint32_t col_s = tmem + kC_ColS + lanes, col_p = tmem + kC_ColP + x * 64 + lanes, col_o = tmem + kC_ColO + x * 128 + lanes;
            const float scale = a.scale_log2 > 0.0f ? a.scale_log2 : 1.0f;   // others are multiplied in beforehand
            uint32_t items = 0, j_phase = 0;             // items of this row tile so far
            // all softmax threads have come this far (bounded, as a barrier of the hardware would not be)
            auto join = [&]() -> bool {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.joint));
                const bool all = wait(sh.joint, j_phase);
                j_phase ^= 1;
                return all;
            };
            bool ok = true;
            for (uint32_t part = 0; ok; ++part) {
                if (!(ok = wait(sh.part_full[part % kC_Parts], (part / kC_Parts) & 1u))) break;
                const volatile ChunkPart &now = sh.parts[part % kC_Parts];   // read where it is needed: registers are for scores
                if (now.toks == 0) break;
                const bool split = now.split;
                const int n_rows = now.toks << a.log2g;
                const int r = split ? row : x * 128 + row;               // row of the unit
                const bool idle = ((split ? 0 : x * 128) + (warp & 3) * 32) >= n_rows;   // no row of this warp exists
                const int rc = r < n_rows ? r : n_rows - 1;              // rows that do not exist follow the last that does
                int limit = now.n;                                    // tokens below it are seen
                if (a.causal) {
                    limit = now.first_pos + (rc >> a.log2g) + 1;
                    if (limit < 0) limit = 0;
                }
                float m = -CUDART_INF_F, l = 0.0f;
                bool any = false;                                        // O holds something
                const int t0 = now.t0, t1 = now.t1;
                for (int j = t0 + (split ? x : 0); j < t1; j += split ? 2 : 1) {
                    if (!(ok = wait(sh.s_full[x], items & 1u))) break;
                    tc_fence_after();
                    if (!idle) {
                        float v[128];
                        load_scores(col_s, v);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh.s_free));
                        const int seen = limit - j * kChunkTile;         // columns below it are seen
                        const bool mask = __any_sync(0xffffffffu, seen < kChunkTile);
                        if (!(a.scale_log2 > 0.0f)) {
#pragma unroll
                            for (int i = 0; i < 128; ++i) v[i] *= a.scale_log2;
                        }
                        if (mask) {
#pragma unroll
                            for (int i = 0; i < 128; ++i)
                                if (i >= seen) v[i] = -CUDART_INF_F;
                        }
                        float x4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                        for (int i = 4; i + 8 <= 124; i += 8) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) x4[k] = max3(x4[k], v[i + k], v[i + 4 + k]);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) x4[k] = fmaxf(x4[k], v[124 + k]);
                        const float mx = max3(x4[0], x4[1], fmaxf(x4[2], x4[3])) * scale;
                        // the last product is done with O and with P
                        if (!(ok = items == 0 || wait(sh.o_done[x], (items - 1) & 1u))) break;
                        tc_fence_after();
                        const bool raise = mx > m + kC_Raise || (m == -CUDART_INF_F && mx > m);
                        if (__any_sync(0xffffffffu, raise)) {
                            const float m_new = raise ? mx : m;
                            const float corr = raise ? exp2_approx(m - m_new) : 1.0f;
                            l *= corr;
                            m = m_new;
                            if (any) {
#pragma unroll 1
                                for (int c = 0; c < 8; ++c) {
                                    uint32_t o[16];
                                    tmem_ld16(col_o + c * 16, o);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
                                    tmem_st16(col_o + c * 16, o);
                                }
                            }
                        }
                        const float base = m == -CUDART_INF_F ? 0.0f : -m;
                        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                float &e0 = v[c * 32 + 2 * i], &e1 = v[c * 32 + 2 * i + 1];
                                fma2(e0, e1, scale, base);
                                e0 = exp2_approx(e0);
                                e1 = exp2_approx(e1);
                                if (i & 1) add2(s2, s3, e0, e1);
                                else add2(s0, s1, e0, e1);
                                pk[i] = pack_bf16(e0, e1);
                            }
                            tmem_st16(col_p + c * 16, pk);
                        }
                        l += (s0 + s1) + (s2 + s3);
                        any = true;
                        tmem_wait_st();
                        tc_fence_before();
                    } else {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&sh.s_free));
                        if (!(ok = items == 0 || wait(sh.o_done[x], (items - 1) & 1u))) break;   // never ahead of the others by more than an item
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[x]));
                    ++items;
                }
                if (!ok || !(ok = items == 0 || wait(sh.o_done[x], (items - 1) & 1u))) break;
                tc_fence_after();

                // ---- join the halves, write the result or this part
                const bool joined = split && t1 - t0 > 1;                // both halves have taken tiles
                float w_own = 1.0f, w_other = 0.0f;
                if (split) {
                    sh.ml[x][row][0] = m;
                    sh.ml[x][row][1] = l;
                    tc_fence_before();
                    if (!(ok = join())) break;
                    tc_fence_after();
                    const float m0 = sh.ml[0][row][0], l0 = sh.ml[0][row][1];
                    const float m1 = joined ? sh.ml[1][row][0] : -CUDART_INF_F, l1 = joined ? sh.ml[1][row][1] : 0.0f;
                    m = fmaxf(m0, m1);
                    const float b = m == -CUDART_INF_F ? 0.0f : m;
                    w_own = exp2_approx(m0 - b);                         // of half 0
                    w_other = exp2_approx(m1 - b);                       // of half 1
                    l = l0 * w_own + (joined ? l1 * w_other : 0.0f);
                }
                // half x of a split unit writes columns 64 x .. 64 x + 63 of the joined row; a row tile of its own all 128
                const int c_lo = split ? 2 * x : 0, c_hi = split ? 2 * x + 2 : 4;
                const bool mine = r < n_rows;
                const long long out_row = ((long long)(now.row + (r >> a.log2g)) * a.Hkv + now.h << a.log2g) + (r & ((1 << a.log2g) - 1));
                const int slot = (int)blockIdx.x * 2 + (now.cut && blockIdx.x == now.first_cta ? 1 : 0);
                const float inv = l > 0.0f ? __frcp_rn(l) : l == 0.0f ? 0.0f : l;   // nothing seen: 0; NaN stays
                if (!idle) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c < c_lo || c >= c_hi) continue;
                        uint32_t v[32];
                        tmem_ld32(tmem + kC_ColO + lanes + (split ? 0 : x * 128) + c * 32, v);
                        tmem_wait_ld();
                        if (split) {
                            if (joined) {
                                uint32_t o[32];
                                tmem_ld32(tmem + kC_ColO + lanes + 128 + c * 32, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    v[i] = __float_as_uint(__uint_as_float(v[i]) * w_own + __uint_as_float(o[i]) * w_other);
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * w_own);
                            }
                        }
                        if (!mine) continue;
                        if (now.wild_v) {              // what was taken out of the V tiles, for the tokens that this row sees
                            const int first = now.first_pos + 1 > 0 ? (now.first_pos + 1) & ~(kChunkTile - 1) : 0, lo = t0 * kChunkTile;
                            const int end = (uint32_t)limit < (uint32_t)t1 * kChunkTile ? limit : t1 * kChunkTile;
                            for (int tok = first > lo ? first : lo; tok < end; ++tok) {
                                const int page = __ldcg(a.table + (long long)now.b * a.bt_sb + (tok >> a.shift));
                                if ((unsigned)page >= (unsigned)a.n_pages) continue;
                                const uint16_t *src = a.V.ptr + (long long)page * a.V.sb + (long long)now.h * a.V.sh + (long long)(tok & ((1 << a.shift) - 1)) * a.V.sn + c * 32;
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const uint32_t w = __ldcg(src + i);
                                    if ((w & 0x7f80u) == 0x7f80u) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w << 16));
                                }
                            }
                        }
                        if (now.cut) {
                            float4 *dst = reinterpret_cast<float4 *>(a.part_acc) + ((long long)slot * (kD / 4) + c * 8) * kChunkRows + r;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                __stcg(dst + i * kChunkRows, make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3])));
                        } else {
                            uint4 *dst = reinterpret_cast<uint4 *>(a.out + out_row * kD + c * 32);
                            uint32_t w[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                w[i] = l == 0.0f ? 0u : pack_bf16(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
                            if ((reinterpret_cast<uintptr_t>(a.out) & 31) == 0) {   // whole sectors of 32 bytes
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 2 * i), "r"(w[8 * i]), "r"(w[8 * i + 1]),
                                                 "r"(w[8 * i + 2]), "r"(w[8 * i + 3]), "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7]) : "memory");
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) dst[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                            }
                        }
                    }
                    if (mine && (!split || x == 0)) {
                        if (now.cut)
                            __stcg(reinterpret_cast<float2 *>(a.part_ml + ((long long)slot * kChunkRows + r) * 2), make_float2(m, l));
                        else if (a.lse)
                            a.lse[out_row] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
                    }
                }
                tc_fence_before();
                bool settle = split;                     // both halves have read both O before the next unit's first product may write them
                if (now.cut) {
                    // ---- the last of the unit's parts joins them
                    __threadfence();
                    if (!(ok = join())) break;
                    if (tid == 0) {
                        const int seen = atomicAdd(a.tickets + now.first_cta, 1);
                        sh.last_part = seen == now.n_parts - 1;
                        if (sh.last_part) a.tickets[now.first_cta] = 0;
                        __threadfence();
                    }
                    if (!(ok = join())) break;
                    if (sh.last_part) {
                        settle = true;                   // ... or what the rows' threads share before the next unit's write it
                        // slot 1 of the first CTA, slot 0 of the others
                        const long long s0 = (long long)now.first_cta * 2 + 1, s1 = (long long)(now.first_cta + 1) * 2;
                        const int np = now.n_parts;
                        auto slot_of = [&](int k) -> long long { return k == 0 ? s0 : s1 + 2 * (k - 1); };
                        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
                        // a row's maximum, and one over its sum, for the threads that share the row
                        auto row_of = [&](int er) -> long long {
                            return ((long long)(now.row + (er >> a.log2g)) * a.Hkv + now.h << a.log2g) + (er & ((1 << a.log2g) - 1));
                        };
                        auto put = [&](int er, float mm, float b, float ll) {
                            sh.joined[er] = make_float2(b, ll == 0.0f ? 0.0f : ll > 0.0f ? __frcp_rn(ll) : ll);
                            if (a.lse) a.lse[row_of(er)] = ll == 0.0f ? -CUDART_INF_F : (mm + log2f(ll)) * kLn2;
                        };
                        if (n_rows <= 32) {            // few rows, which may have many parts: a lane for each part
                            for (int er = warp; er < n_rows; er += kC_Softmax / 32) {
                                float mm = -CUDART_INF_F, ll = 0.0f;
                                for (int k = lane; k < np; k += 32) {
                                    const float2 v = __ldcg(&ml[slot_of(k) * kChunkRows + er]);
                                    const float m_new = fmaxf(mm, v.x), base = m_new == -CUDART_INF_F ? 0.0f : m_new;
                                    ll = fmaf(ll, exp2_approx(mm - base), v.y * exp2_approx(v.x - base));
                                    mm = m_new;
                                }
                                float top = mm;
#pragma unroll
                                for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                                const float b = top == -CUDART_INF_F ? 0.0f : top;
                                ll *= exp2_approx(mm - b);
#pragma unroll
                                for (int d = 16; d > 0; d >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, d);
                                if (lane == 0) put(er, top, b, ll);
                            }
                        } else if (tid < n_rows) {
                            float mm = -CUDART_INF_F, ll = 0.0f;
#pragma unroll 4
                            for (int k = 0; k < np; ++k) mm = fmaxf(mm, __ldcg(&ml[slot_of(k) * kChunkRows + tid]).x);
                            const float b = mm == -CUDART_INF_F ? 0.0f : mm;
#pragma unroll 4
                            for (int k = 0; k < np; ++k) {
                                const float2 v = __ldcg(&ml[slot_of(k) * kChunkRows + tid]);
                                ll = fmaf(v.y, exp2_approx(v.x - b), ll);
                            }
                            put(tid, mm, b, ll);
                        }
                        if (!(ok = join())) break;
                        // A thread takes kU pieces of eight columns of a row at a time, and kK parts of them: all of those loads are in flight
                        const int lrows = 32 - __clz(n_rows - 1 > 0 ? n_rows - 1 : 1), rows2 = 1 << lrows;   // rows, rounded up to a power of two
                        auto join_parts = [&](auto u_, auto k_) {
                            constexpr int kU = decltype(u_)::value, kK = decltype(k_)::value;
                            for (int e0 = tid; e0 < 16 * rows2; e0 += kU * kC_Softmax) {
                                float acc[kU][8];
#pragma unroll
                                for (int u = 0; u < kU; ++u)
#pragma unroll
                                    for (int i = 0; i < 8; ++i) acc[u][i] = 0.0f;
                                for (int k0 = 0; k0 < np; k0 += kK) {
                                    float4 v[kU][kK][2];
                                    float mk[kU][kK];
#pragma unroll
                                    for (int u = 0; u < kU; ++u) {
                                        const int e = e0 + u * kC_Softmax, er = e & (rows2 - 1), ec = e >> lrows;
#pragma unroll
                                        for (int k = 0; k < kK; ++k) {
                                            v[u][k][0] = v[u][k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
                                            mk[u][k] = -CUDART_INF_F;
                                            if (ec >= 16 || er >= n_rows || k0 + k >= np) continue;
                                            const long long sl = slot_of(k0 + k);
                                            const float4 *src = reinterpret_cast<const float4 *>(a.part_acc) + (sl * (kD / 4) + 2 * ec) * kChunkRows + er;
                                            v[u][k][0] = __ldcg(src);
                                            v[u][k][1] = __ldcg(src + kChunkRows);
                                            mk[u][k] = __ldcg(&ml[sl * kChunkRows + er]).x;
                                        }
                                    }
#pragma unroll
                                    for (int u = 0; u < kU; ++u) {
                                        const float b = sh.joined[(e0 + u * kC_Softmax) & (rows2 - 1)].x;
#pragma unroll
                                        for (int k = 0; k < kK; ++k) {
                                            const float w = exp2_approx(mk[u][k] - b);
#pragma unroll
                                            for (int i = 0; i < 2; ++i) {
                                                acc[u][4 * i] = fmaf(v[u][k][i].x, w, acc[u][4 * i]);
                                                acc[u][4 * i + 1] = fmaf(v[u][k][i].y, w, acc[u][4 * i + 1]);
                                                acc[u][4 * i + 2] = fmaf(v[u][k][i].z, w, acc[u][4 * i + 2]);
                                                acc[u][4 * i + 3] = fmaf(v[u][k][i].w, w, acc[u][4 * i + 3]);
                                            }
                                        }
                                    }
                                }
#pragma unroll
                                for (int u = 0; u < kU; ++u) {
                                    const int e = e0 + u * kC_Softmax, er = e & (rows2 - 1), ec = e >> lrows;
                                    if (ec >= 16 || er >= n_rows) continue;
                                    const float inv = sh.joined[er].y;
                                    uint4 w = make_uint4(0u, 0u, 0u, 0u);
                                    if (inv != 0.0f)
                                        w = make_uint4(pack_bf16(acc[u][0] * inv, acc[u][1] * inv), pack_bf16(acc[u][2] * inv, acc[u][3] * inv),
                                                       pack_bf16(acc[u][4] * inv, acc[u][5] * inv), pack_bf16(acc[u][6] * inv, acc[u][7] * inv));
                                    *reinterpret_cast<uint4 *>(a.out + row_of(er) * kD + ec * 8) = w;
                                }
                            }
                        };
                        if (n_rows <= 32) join_parts(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
                        else join_parts(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
                    }
                }
                if (settle) ok = join();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// ---- workspace: front (the tickets in it), parts
size_t chunk_workspace_bytes() {
    return kWorkspaceFront + (size_t)2 * kChunkMaxCtas * kChunkRows * (2 + kD) * 4;
}

// Tensor maps (bf16, strides in elements): q [n_rows][Hq][128] and a pool [n_pages][Hkv][page][128], both with the 128 columns as two
// halves of 64; false if the driver's encoder is missing or the strides do not fit a tensor map.
static bool encode_map(CUtensorMap *tm, int rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box) {
    const cuuint32_t step[5] = {1u, 1u, 1u, 1u, 1u};
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    for (int i = 0; i < rank; ++i)
        if (dims[i] == 0 || dims[i] > (1ull << 32) || (i + 1 < rank && (strides[i] == 0 || (strides[i] & 15) || strides[i] >= (1ull << 40)))) return false;
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static bool q_map(CUtensorMap *tm, TensorView q, int rows, int Hq, int log2g) {
    const cuuint64_t dims[4] = {64u, (cuuint64_t)Hq, (cuuint64_t)rows, 2u};
    const cuuint64_t strides[3] = {(cuuint64_t)q.sh * 2, (cuuint64_t)q.sn * 2, 128u};
    const cuuint32_t box[4] = {64u, 1u << log2g, (cuuint32_t)(kChunkTile >> log2g), 2u};
    return encode_map(tm, 4, q.ptr, dims, strides, box);
}
static bool pool_map(CUtensorMap *tm, TensorView T, int n_pages, int Hkv, int shift, int log2box, int halves) {
    const cuuint64_t dims[5] = {64u, 1ull << shift, 2u, (cuuint64_t)Hkv, (cuuint64_t)n_pages};
    const cuuint64_t strides[4] = {(cuuint64_t)T.sn * 2, 128u, (cuuint64_t)T.sh * 2, (cuuint64_t)T.sb * 2};
    const cuuint32_t box[5] = {64u, 1u << log2box, (cuuint32_t)halves, 1u, 1u};
    return encode_map(tm, 5, T.ptr, dims, strides, box);
}

cudaError_t launch_chunk_attn(int B, int Hq, int Hkv, float sm_scale, TensorView q, const int32_t *offsets, int n_rows, TensorView K,
                              TensorView V, int n_pages, const int32_t *table, long long bt_sb, int shift, const int32_t *seq_lens,
                              bool causal, uint16_t *out, float *lse, void *workspace, cudaStream_t st) {
    ChunkArgs a;
    a.q = q.ptr; a.q_sn = q.sn; a.q_sh = q.sh;
    a.offsets = offsets; a.seq_lens = seq_lens; a.table = table;
    a.K = K; a.V = V; a.bt_sb = bt_sb;
    a.n_rows = n_rows; a.n_pages = n_pages; a.shift = shift; a.B = B; a.Hkv = Hkv; a.causal = causal;
    a.log2g = 0;
    while ((Hkv << a.log2g) < Hq) ++a.log2g;
    a.max_ctas = kChunkMaxCtas;
    a.log2box = shift < 7 ? shift : 7;
    a.scale_log2 = sm_scale * kLog2e;
    a.out = out; a.lse = lse;
    char *ws = reinterpret_cast<char *>(workspace);
    a.status = reinterpret_cast<uint32_t *>(ws);
    a.tickets = reinterpret_cast<int32_t *>(ws + kOffChunkTickets);
    a.part_ml = reinterpret_cast<float *>(ws + kWorkspaceFront);
    a.part_acc = a.part_ml + (size_t)2 * kChunkMaxCtas * kChunkRows * 2;
    CUtensorMap mq, mk, mv;
    memset(&mq, 0, sizeof(mq));
    memset(&mk, 0, sizeof(mk));
    memset(&mv, 0, sizeof(mv));
    const bool tma = shift >= 3 && q_map(&mq, q, n_rows, Hq, a.log2g) && pool_map(&mk, K, n_pages, Hkv, shift, a.log2box, 1) &&
                     pool_map(&mv, V, n_pages, Hkv, shift, a.log2box, 2);
    cudaError_t e = cudaFuncSetAttribute(tma ? chunk_attn_kernel<true> : chunk_attn_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kC_Smem);
    if (e != cudaSuccess) return e;
    int grid = sm_count();
    if (grid > kChunkMaxCtas) grid = kChunkMaxCtas;
    e = launch_pdl(tma ? chunk_attn_kernel<true> : chunk_attn_kernel<false>, dim3(grid), dim3(kC_Threads), kC_Smem, st, mq, mk, mv, a);
    if (e != cudaSuccess) return e;
    count_launch();
    return cudaGetLastError();
}

} // namespace ha
