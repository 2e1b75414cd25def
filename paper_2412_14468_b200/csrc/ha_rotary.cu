// Rotary positions, and the new tokens' way into the paged cache.
//
// Pair (x, y) of a head's first rot_dim values at position p is turned by the angle p w_i:
//     (x, y) -> scale (x cos - y sin, x sin + y cos)
// with (x, y) = values (i, i + rot_dim / 2), or (2 i, 2 i + 1) interleaved; `inverse` turns by the negative angle, which is the
// gradient's way back.  The rest of the head passes through.
//
// The angle of a far position needs more than 32 bits: p w reduced to one turn.  w / (2 pi) is taken as a 64-bit fraction of a turn,
// so that p times it, modulo 2^64, is the reduced angle exactly (two integer multiplications); what is left of the frequency's own
// rounding is p w 2^-53.  The top bits become a float for sincospif.
//
// What bounds it: HBM (a row of 256 bytes is read and written once), and for a few tokens the launch and two dependent loads.
// Measured: 22 400 new tokens of 32 + 8 + 8 heads appended in 95 us (5.8 TB/s), 64 in 4.7; 5001 rows of 32 heads turned in 17 (4.8 TB/s).
// Loads go past L1, which may hold what was there before a kernel in front wrote (see the note on programmatic launches), but for the
// frequencies, which all threads share (through L2 alone 95 -> 139 us).
// Eight lanes hold the cosines and sines of a token (eight pairs each, once for all its heads) and take its heads one after the
// other, 16 values at a time; the four such groups of a warp take every fourth head.
#include "ha_common.cuh"
#include "ha_attn_dev.cuh"

namespace ha {

constexpr int kR_Threads = 128;

struct RotaryTurn {
    const double *inv_freq;       // radians per position, [rot_dim / 2]
    int half;                     // rot_dim / 2, a multiple of 8
    bool interleaved, inverse;
    float scale;
};
struct RotaryRows {               // bf16 rows [rows][heads][128]
    const uint16_t *src;
    long long s_sn, s_sh;
    uint16_t *dst;
    long long d_sn, d_sh;
};
struct RotaryArgs {
    RotaryTurn turn;
    const int32_t *positions;     // [rows], or NULL: the place in the cache
    int rows, heads, warps_per_row;
    RotaryRows x;                 // what is turned: x, or q
    // the new tokens' way into the cache (kAppend)
    const uint16_t *k, *v;
    long long k_sn, k_sh, v_sn, v_sh;
    uint16_t *k_out;              // [rows][kv_heads][128] contiguous or NULL
    const int32_t *offsets, *seq_lens, *table;
    TensorView K, V;
    long long bt_sb;
    int B, kv_heads, n_pages, shift;
    uint32_t *status;
};

// cos and sin (scaled) of this lane's eight pairs at position p
__device__ __forceinline__ void rotary_angles(const RotaryTurn &t, int first, int p, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = 1.0f;
        s[i] = 0.0f;
    }
    if (first >= t.half) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        double f = __ldg(t.inv_freq + first + i) * 0.15915494309189533577;   // turns per position
        f -= floor(f);
        const unsigned long long turn = (unsigned long long)(long long)p * __double2ull_rn(f * 18446744073709551616.0);
        const float half_turns = __ll2float_rn((long long)turn) * 1.0842021724855044e-19f;   // 2^-63: in [-1, 1]
        float sn, cs;
        sincospif(half_turns, &sn, &cs);
        c[i] = cs * t.scale;
        s[i] = (t.inverse ? -sn : sn) * t.scale;
    }
}

__device__ __forceinline__ float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// What lane `piece` (0 .. 7) has of a row: two runs of 8 values.  Half layout: values 8 piece .. of either half; interleaved: the
// 16 values of pairs 8 piece ..; values behind the turned ones: 16 in a row.
__device__ __forceinline__ void rotary_places(const RotaryTurn &t, int piece, int &a, int &b) {
    const int turned = t.half / 8;      // lanes that turn
    if (piece < turned && !t.interleaved) {
        a = piece * 8;
        b = t.half + a;
    } else {
        a = piece * 16;
        b = a + 8;
    }
}
__device__ __forceinline__ void rotary_apply(const RotaryTurn &t, bool turns, const float (&c)[8], const float (&s)[8], uint4 &a, uint4 &b) {
    if (!turns) return;
    uint32_t va[4] = {a.x, a.y, a.z, a.w}, vb[4] = {b.x, b.y, b.z, b.w};
    if (t.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = lo_f(va[i]), y0 = hi_f(va[i]), x1 = lo_f(vb[i]), y1 = hi_f(vb[i]);
            va[i] = pack_bf16(x0 * c[i] - y0 * s[i], x0 * s[i] + y0 * c[i]);
            vb[i] = pack_bf16(x1 * c[4 + i] - y1 * s[4 + i], x1 * s[4 + i] + y1 * c[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = lo_f(va[i]), x1 = hi_f(va[i]), y0 = lo_f(vb[i]), y1 = hi_f(vb[i]);
            va[i] = pack_bf16(x0 * c[2 * i] - y0 * s[2 * i], x1 * c[2 * i + 1] - y1 * s[2 * i + 1]);
            vb[i] = pack_bf16(x0 * s[2 * i] + y0 * c[2 * i], x1 * s[2 * i + 1] + y1 * c[2 * i + 1]);
        }
    }
    a = make_uint4(va[0], va[1], va[2], va[3]);
    b = make_uint4(vb[0], vb[1], vb[2], vb[3]);
}

// The last b with offsets[b] <= row, of ascending offsets; 32 offsets are looked at a time.  -1: none.
__device__ __forceinline__ int sequence_of(const int32_t *offsets, int B, int row, int lane) {
    int lo = 0, n = B + 1;                // offsets[lo .. lo + n) are left, all in front of lo are <= row
    for (;;) {
        const int step = (n + 31) / 32, i = lo + lane * step;
        const bool le = lane * step < n && __ldcg(offsets + i) <= row;
        const uint32_t m = __ballot_sync(0xffffffffu, le);
        if (m == 0) return -1;            // only in the first round: row lies in front of the first
        const int at = 31 - __clz(m);
        const int first = lo + at * step;
        if (step == 1) return first < B ? first : -1;
        n = n - at * step < step ? n - at * step : step;
        lo = first;
    }
}

__device__ __forceinline__ bool offsets_in_order(const int32_t *offsets, int b, int rows, int &o0, int &o1) {
    o0 = __ldcg(offsets + b);
    o1 = __ldcg(offsets + b + 1);
    return o0 >= 0 && o1 >= o0 && o1 <= rows;
}
// The sequence that row belongs to, and its offsets; -1: none.  Where offsets are not ascending the search may miss the sequence that has
// the row, so a row that it finds no place for is looked for in every sequence (as are the rows behind the last one: a load a lane for
// every 32 sequences).
__device__ __forceinline__ int owner_of(const int32_t *offsets, int B, int rows, int row, int lane, int &o0, int &o1) {
    int b = sequence_of(offsets, B, row, lane);
    if (b >= 0 && offsets_in_order(offsets, b, rows, o0, o1) && row >= o0 && row < o1) return b;
    for (int b0 = 0; b0 < B; b0 += 32) {
        b = b0 + lane;
        const bool mine = b < B && offsets_in_order(offsets, b, rows, o0, o1) && row >= o0 && row < o1;
        const uint32_t m = __ballot_sync(0xffffffffu, mine);
        if (m) {
            b = b0 + __ffs(m) - 1;
            offsets_in_order(offsets, b, rows, o0, o1);
            return b;
        }
    }
    return -1;
}

template <bool kAppend>
__global__ void __launch_bounds__(kR_Threads) rotary_kernel(const RotaryArgs a) {
    const int lane = threadIdx.x & 31, piece = lane & 7, group = lane >> 3;
    const long long unit = ((long long)blockIdx.x * kR_Threads + threadIdx.x) >> 5;
    const int row = (int)(unit / a.warps_per_row), part = (int)(unit % a.warps_per_row);
    pdl_wait();
    pdl_launch_dependents();   // no kernel reads what is written here before its own wait
    if (kAppend && a.status && blockIdx.x == gridDim.x - 1) {   // a CTA behind those of the rows
        int o0, o1;
        bool bad = false;
        for (int b = threadIdx.x; b < a.B; b += kR_Threads) bad |= !offsets_in_order(a.offsets, b, a.rows, o0, o1);
        if (bad) atomicOr(a.status, HA_DEV_BAD_INDEX);
        return;
    }
    if (row >= a.rows) return;

    int pos;
    long long k_at = -1, v_at = -1;
    // No room was made for the new tokens: the places that seq_lens gives them are those of tokens cached earlier, which stay.  k_out then
    // holds those tokens' keys, so that a signature made of it is the one that is there.
    bool refused = false;
    if (kAppend) {
        refused = a.status && __ldcg(a.status + kRefusedWord) != 0u;
        int o0, o1;
        const int b = owner_of(a.offsets, a.B, a.rows, row, lane, o0, o1);
        if (b < 0) return;                // of no sequence
        const int tok = __ldcg(a.seq_lens + b) - o1 + row;
        pos = a.positions ? __ldcg(a.positions + row) : tok;
        if (tok >= 0) {
            const int page = __ldcg(a.table + (long long)b * a.bt_sb + (tok >> a.shift));
            if ((unsigned)page < (unsigned)a.n_pages) {
                const long long slot = tok & ((1 << a.shift) - 1);
                k_at = (long long)page * a.K.sb + slot * a.K.sn;
                v_at = (long long)page * a.V.sb + slot * a.V.sn;
            } else if (a.status && lane == 0) atomicOr(a.status, HA_DEV_BAD_INDEX);
        }
    } else {
        pos = __ldcg(a.positions + row);
    }

    const int turned = a.turn.half / 8;
    const bool turns = piece < turned;
    int pa, pb;
    rotary_places(a.turn, piece, pa, pb);
    float c[8], s[8];
    rotary_angles(a.turn, piece * 8, pos, c, s);

    const int heads = kAppend ? a.heads + 2 * a.kv_heads : a.heads;
    for (int h = part * 4 + group; h < heads; h += 4 * a.warps_per_row) {
        const uint16_t *src;
        uint16_t *dst, *also = nullptr;
        bool turn = turns;
        if (!kAppend || h < a.heads) {
            src = a.x.src + (long long)row * a.x.s_sn + (long long)h * a.x.s_sh;
            dst = a.x.dst + (long long)row * a.x.d_sn + (long long)h * a.x.d_sh;
        } else if (h < a.heads + a.kv_heads) {
            const int g = h - a.heads;
            src = a.k + (long long)row * a.k_sn + (long long)g * a.k_sh;
            dst = k_at < 0 ? nullptr : const_cast<uint16_t *>(a.K.ptr) + k_at + (long long)g * a.K.sh;
            if (refused && dst) {
                src = dst;
                dst = nullptr;
                turn = false;
            }
            if (a.k_out) also = a.k_out + ((long long)row * a.kv_heads + g) * kD;
        } else {
            const int g = h - a.heads - a.kv_heads;
            src = a.v + (long long)row * a.v_sn + (long long)g * a.v_sh;
            dst = v_at < 0 || refused ? nullptr : const_cast<uint16_t *>(a.V.ptr) + v_at + (long long)g * a.V.sh;
            turn = false;
        }
        uint4 va = __ldcg(reinterpret_cast<const uint4 *>(src + pa)), vb = __ldcg(reinterpret_cast<const uint4 *>(src + pb));
        rotary_apply(a.turn, turn, c, s, va, vb);
        if (dst) {
            *reinterpret_cast<uint4 *>(dst + pa) = va;
            *reinterpret_cast<uint4 *>(dst + pb) = vb;
        }
        if (also) {
            *reinterpret_cast<uint4 *>(also + pa) = va;
            *reinterpret_cast<uint4 *>(also + pb) = vb;
        }
    }
}

// Warps of a row: one where the rows fill the GPU, else as many as take one head a group each.
static int rotary_warps_per_row(int rows, int heads) {
    const int most = (heads + 3) / 4;
    const long long want = (long long)sm_count() * 16;
    long long w = want / (rows > 0 ? rows : 1);
    if (w < 1) w = 1;
    return w < most ? (int)w : most;
}

template <bool kAppend>
static cudaError_t launch_rotary_kernel(const RotaryArgs &a, int heads, cudaStream_t st) {
    const long long warps = (long long)a.rows * a.warps_per_row;
    const dim3 grid((unsigned)((warps * 32 + kR_Threads - 1) / kR_Threads) + (kAppend && a.status ? 1u : 0u));
    const cudaError_t e = launch_pdl(rotary_kernel<kAppend>, grid, dim3(kR_Threads), 0, st, a);
    if (e != cudaSuccess) return e;
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_rotary(TensorView x, TensorView y, int rows, int heads, const double *inv_freq, int rot_dim, const int32_t *positions,
                          bool interleaved, bool inverse, float scale, cudaStream_t st) {
    RotaryArgs a = {};
    a.turn = RotaryTurn{inv_freq, rot_dim / 2, interleaved, inverse, scale};
    a.positions = positions;
    a.rows = rows; a.heads = heads;
    a.warps_per_row = rotary_warps_per_row(rows, heads);
    a.x = RotaryRows{x.ptr, x.sn, x.sh, const_cast<uint16_t *>(y.ptr), y.sn, y.sh};
    return launch_rotary_kernel<false>(a, heads, st);
}

cudaError_t launch_rotary_append(int B, int Hq, int Hkv, TensorView q, TensorView k, TensorView v, TensorView q_out, uint16_t *k_out,
                                 const int32_t *offsets, int rows, const double *inv_freq, int rot_dim, const int32_t *positions,
                                 bool interleaved, float scale, TensorView K, TensorView V, int n_pages, const int32_t *table,
                                 long long bt_sb, int shift, const int32_t *seq_lens, uint32_t *status, cudaStream_t st) {
    RotaryArgs a = {};
    a.turn = RotaryTurn{inv_freq, rot_dim / 2, interleaved, false, scale};
    a.positions = positions;
    a.rows = rows; a.heads = Hq;
    a.warps_per_row = rotary_warps_per_row(rows, Hq + 2 * Hkv);
    a.x = RotaryRows{q.ptr, q.sn, q.sh, const_cast<uint16_t *>(q_out.ptr), q_out.sn, q_out.sh};
    a.k = k.ptr; a.k_sn = k.sn; a.k_sh = k.sh;
    a.v = v.ptr; a.v_sn = v.sn; a.v_sh = v.sh;
    a.k_out = k_out;
    a.offsets = offsets; a.seq_lens = seq_lens; a.table = table;
    a.K = K; a.V = V; a.bt_sb = bt_sb;
    a.B = B; a.kv_heads = Hkv; a.n_pages = n_pages; a.shift = shift;
    a.status = status;
    return launch_rotary_kernel<true>(a, Hq + 2 * Hkv, st);
}

} // namespace ha
