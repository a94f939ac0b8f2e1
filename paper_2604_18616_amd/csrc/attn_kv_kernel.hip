// Attention over the quantised paged cache, gfx950.
//
// The query rows that share a kv head (g = Hq / Hkv heads x Sq positions, the g heads of a position side by side) are packed
// into blocks of 16, the columns of v_mfma_f32_16x16x32_bf16: S^T = K Q^T, O^T += V^T P^T, so that a row's running maximum
// and sum are scalars of a lane.  A wavefront walks tiles of 64 keys on its own, straight from memory into registers, without
// LDS and without barriers:
//   * K: a lane reads 16 consecutive codes of its key, two steps of the matrix instruction (the order of the sum over d is
//     free as long as Q is read in the same one);
//   * row m of key block t of a tile stands for key 16 (m / 4) + 4 t + m % 4, so that after four blocks lane group l / 16
//     holds the scores of 16 consecutive keys: the same 16 keys whose codes of one d are one 16-byte load of the transposed V;
//   * codes become bf16, exactly and times the page's scale, by the conversion instruction; 16 keys lie in one page, so the
//     scale and the page's address are per lane.
// The keys are cut over the wavefronts of a workgroup and over `splits` workgroups; the wavefronts are merged through LDS,
// the workgroups of a row by attn_kv_combine from fp32 parts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "kv_launch.h"

namespace {

using namespace gfx950;

constexpr int kTile = 64;            // keys per tile
constexpr int kBlock = 16;           // packed query rows per block

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// What the rows of a workgroup see of a sequence: tiles 0 ... sink_tiles - 1 and first ... first + count - sink_tiles - 1.
struct Seen { int n, rows, pos0, count, sink_tiles, first; };
__device__ __forceinline__ Seen seen_tiles(const KvAttnParams& p, int b, int g, int first_row, int rows_per_wg) {
    Seen s;
    s.n = min(max(p.lens[b], 0), p.max_len);
    s.rows = p.q_lens ? min(max(p.q_lens[b], 0), p.Sq) : p.Sq;
    s.pos0 = s.n - s.rows;                                   // position of query row 0
    const int i0 = first_row / g, i1 = min((first_row + rows_per_wg - 1) / g, s.rows - 1);
    s.count = s.sink_tiles = s.first = 0;
    if (i0 > i1 || s.n == 0) return s;
    const int last = p.causal ? min(s.n - 1, s.pos0 + i1) : s.n - 1;
    if (last < 0) return s;
    const long long low = p.window ? (long long)s.pos0 + i0 - p.window + 1 : 0;
    s.first = low > 0 ? (int)(low / kTile) : 0;
    s.sink_tiles = min(s.first, (int)(((long long)min(p.sinks, last + 1) + kTile - 1) / kTile));
    s.count = s.sink_tiles + max(last / kTile + 1 - s.first, 0);
    return s;
}

// Tiles of a part.  All sequences' parts have one size, by the longest of them: the workgroups of a batch with caches of all
// lengths then take equally long.  (Never so few that a sequence had more parts than there is room for.)
__device__ __forceinline__ int part_tiles(const KvAttnParams& p, const Seen& seen, int lane) {
    if (p.splits == 1) return seen.count;
    int longest = seen.n;
    if (p.B > 1) {
        for (int x = lane; x < p.B; x += 64) longest = max(longest, p.lens[x]);
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) longest = max(longest, __shfl_xor(longest, x));
    }
    const int tiles = max(min((min(__builtin_amdgcn_readfirstlane(longest), p.max_len) + kTile - 1) / kTile, p.most_tiles), seen.count);
    return (tiles + p.splits - 1) / p.splits;
}

// The largest or the sum over the four lane groups that share a column.
__device__ __forceinline__ float max_over_groups(float x) { x = fmaxf(x, __shfl_xor(x, 16)); return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float sum_over_groups(float x) { x += __shfl_xor(x, 16); return x + __shfl_xor(x, 32); }

// Eight codes (two dwords) as a matrix operand, times 2^e (scale: 2^e as fp32).
__device__ __forceinline__ bf16x8 decode(unsigned lo, unsigned hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The bytes of w that are the NaN code, as 0x80 each.
__device__ __forceinline__ unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A part without keys: its rows' maxima say so, its O stays unwritten.
template <int ROWS>
__device__ __forceinline__ void no_part(const KvAttnParams& p, int b, int hk, int g, int first, int split) {
    const int row = first + (int)threadIdx.x, i = row / g, h = row - i * g;
    if (threadIdx.x < ROWS && i < p.Sq)
        *(f32x2*)(p.ml + 2 * ((((size_t)b * p.Hq + hk * g + h) * p.Sq + i) * p.splits + split)) = f32x2{-INFINITY, 0.f};
}

template <int D> constexpr int merge_pitch() { return D + 4; }      // floats per O row in the merge area

// NR blocks of 16 packed rows per workgroup, every wavefront all of them.
template <int D, int NR, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv_rows(KvAttnParams p) {
    constexpr int KC = D / 64;                 // 16-byte loads per key and lane
    constexpr int DT = D / 16;                 // 16-row blocks of O^T
    constexpr int PITCH = merge_pitch<D>();
    constexpr int ROWS = NR * kBlock;

    __shared__ __attribute__((aligned(16))) float s_o[NW * ROWS * PITCH];
    __shared__ float s_ml[2][NW][ROWS];
    __shared__ float s_inv[ROWS];

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Workgroup id -> (kv head of a sequence, split, row block); every XCD takes a contiguous range, so that row blocks of one
    // split, which read the same keys, share an L2.
    const int nb = gridDim.x, per_xcd = nb >> 3, bid = blockIdx.x;
    int logical = bid < per_xcd * 8 ? (bid & 7) * per_xcd + (bid >> 3) : bid;
    const int rowblk = logical % p.row_wgs; logical /= p.row_wgs;
    const int split = logical % p.splits; logical /= p.splits;
    const int B = p.B, b = logical % B, hk = logical / B;                // (an XCD gets heads, and so sequences of all lengths)

    const int g = p.Hq / p.c.Hkv, R = g * p.Sq, first = rowblk * ROWS;
    const Seen seen = seen_tiles(p, b, g, first, ROWS);
    const int per = part_tiles(p, seen, lane);
    const int t0 = split * per, t1 = min(seen.count, t0 + per);
    const bool alone = p.splits == 1;                        // the result itself, no part of it
    if (!alone && t0 >= t1) { no_part<ROWS>(p, b, hk, g, first, split); return; }

    // this lane's rows: what they see, and Q.  Rows past the last one see what the last one does and are not stored.
    int hi[NR], lo[NR];
    bf16x8 qf[NR][KC * 2];
    int hi_all = -1, lo_all = INT_MAX;                       // what any row of the workgroup sees
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = min(first + r * kBlock + col, R - 1), i = min(row / g, max(seen.rows - 1, 0)), h = row - row / g * g;
        const int pos = seen.pos0 + i;
        hi[r] = p.causal ? min(pos, seen.n - 1) : seen.n - 1;
        lo[r] = p.window ? (int)max((long long)pos - p.window + 1, 0LL) : 0;
        hi_all = max(hi_all, hi[r]); lo_all = min(lo_all, lo[r]);
        const __bf16* const q = p.q + b * p.q_sb + (hk * g + h) * p.q_sh + (long long)(row / g) * p.q_ss;      // (not i: no wait for the lengths)
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) qf[r][2 * c + u] = *(const bf16x8*)(q + (grp + 4 * c) * 16 + 8 * u);
    }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) { hi_all = max(hi_all, __shfl_xor(hi_all, x)); lo_all = min(lo_all, __shfl_xor(lo_all, x)); }

    f32x4 oacc[NR][DT];
    float m_run[NR], l_run[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m_run[r] = -INFINITY; l_run[r] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) oacc[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float c = p.scale_log2;
    const int page = p.c.page, sub_k = col >> 2, key_k = col & 3;
    const int* const table = p.c.table + b * p.c.pitch;
    bool poisoned = false;                                   // NaN codes were met where only some rows see them

    auto tile_of = [&](int t) __attribute__((always_inline)) { return t < seen.sink_tiles ? t : t - seen.sink_tiles + seen.first; };
    // the pages of this lane's keys in a tile, for K and for V: -1 where there is none
    struct Pages { int k, v; };
    auto lookup = [&](int key) __attribute__((always_inline)) {
        const int at = table[min(key, seen.n - 1) >> p.c.page_log2];           // (no branch around the load: several are in flight)
        return (int)(key < seen.n) & (int)((unsigned)at < (unsigned)p.c.P) ? at : -1;
    };
    auto find = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(t) * kTile;
        return Pages{lookup(key0 + 16 * sub_k), lookup(key0 + 16 * grp)};
    };
    // Loads of a tile's codes.  Behind the last tile every lane reads the cache's first bytes instead: the number of loads in
    // flight, which the waits count, is the same on every path.
    u32x4 kr[4][KC], vr[DT];
    unsigned ke, ve;
    int at_v;
    auto load_k = [&](int t, int at) __attribute__((always_inline)) {
        const size_t unit = (size_t)max(at, 0) * p.c.Hkv + hk;
        const unsigned char* k = p.c.k + (unit * page + ((tile_of(t) * kTile + 16 * sub_k) & (page - 1)) + key_k) * D + 16 * grp;
        k = t < t1 ? k : p.c.k;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int ch = 0; ch < KC; ++ch) kr[kt][ch] = *(const u32x4*)(k + 4 * kt * D + 64 * ch);
        ke = p.c.ke[unit];
    };
    auto load_v = [&](int t, int at) __attribute__((always_inline)) {
        const size_t unit = (size_t)max(at, 0) * p.c.Hkv + hk;
        const unsigned char* v = p.c.v + unit * page * D + col * page + ((tile_of(t) * kTile + 16 * grp) & (page - 1));
        v = t < t1 ? v : p.c.v;
#pragma unroll
        for (int d = 0; d < DT; ++d) vr[d] = *(const u32x4*)(v + d * 16 * page);
        ve = p.c.ve[unit];
        at_v = at;
    };
    // which of this lane's 16 keys from `key` on a row sees whose last key is hi and whose window starts at lo
    auto sees = [&](int key, int hi, int lo, bool there) __attribute__((always_inline)) {
        auto upto = [](int n) __attribute__((always_inline)) { return (1u << min(max(n, 0), 16)) - 1; };
        return there ? upto(hi - key + 1) & (~upto(lo - key) | upto(p.sinks - key)) : 0u;
    };
    // a tile with keys that some row does not see
    auto at_edge = [&](int key0, int at_v) __attribute__((always_inline)) {
        bool edge = at_v < 0;
#pragma unroll
        for (int r = 0; r < NR; ++r) edge = edge || key0 + kTile - 1 > hi[r] || (key0 < lo[r] && key0 + kTile > p.sinks);
        return __builtin_amdgcn_ballot_w64(edge) != 0;
    };

    f32x4 sc[NR][4];
    bf16x8 pf[NR][2];
    auto scores = [&]() __attribute__((always_inline)) {
        const float scale = __uint_as_float(ke << 23);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int r = 0; r < NR; ++r) sc[r][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ch = 0; ch < KC; ++ch)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bf16x8 kf = decode(kr[kt][ch][2 * u], kr[kt][ch][2 * u + 1], scale);
#pragma unroll
                    for (int r = 0; r < NR; ++r) sc[r][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][2 * ch + u], sc[r][kt], 0, 0, 0);
                }
        }
    };
    auto softmax = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(t) * kTile;
        if (at_edge(key0, at_v)) {
            const int key = key0 + 16 * grp;                 // this lane's scores are those of 16 keys from here on
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const unsigned visible = sees(key, hi[r], lo[r], at_v >= 0);
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[r][j / 4][j % 4] = visible >> j & 1 ? sc[r][j / 4][j % 4] : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float mx = sc[r][0][0];
#pragma unroll
            for (int j = 1; j < 16; ++j) mx = fmaxf(mx, sc[r][j / 4][j % 4]);
            const float m_new = fmaxf(m_run[r], max_over_groups(mx));
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2_hw((m_run[r] - m_use) * c), mc = m_use * c;
            m_run[r] = m_new;
            float sum = 0.f;
            unsigned pk[8];
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float p0 = exp2_hw(fmaf(sc[r][j / 4][j % 4], c, -mc)), p1 = exp2_hw(fmaf(sc[r][j / 4][j % 4 + 1], c, -mc));
                sum += p0 + p1;
                pk[j / 2] = pack_bf16x2(p0, p1);
            }
            l_run[r] = l_run[r] * alpha + sum;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0)
#pragma unroll
                for (int d = 0; d < DT; ++d) oacc[r][d] *= alpha;
            pf[r][0] = __builtin_bit_cast(bf16x8, (u32x4{pk[0], pk[1], pk[2], pk[3]}));
            pf[r][1] = __builtin_bit_cast(bf16x8, (u32x4{pk[4], pk[5], pk[6], pk[7]}));
        }
    };
    auto weigh = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(t) * kTile;
        const float scale = __uint_as_float(ve << 23);
        if (at_edge(key0, at_v)) {
            // NaN codes become zero: the probability 0 of a row that does not see them must not meet them
            const unsigned some = sees(key0 + 16 * grp, hi_all, lo_all, at_v >= 0);
            unsigned bad = 0;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned nan = nan_codes(vr[d][j]) >> 7;
                    vr[d][j] &= ~(nan * 0xffu);
                    bad |= (nan * 0x10204080u >> 28) << (4 * j);                      // bytes 0 ... 3 to bits 0 ... 3
                }
            poisoned = poisoned || __builtin_amdgcn_ballot_w64((bad & some) != 0) != 0;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 vf = decode(vr[d][2 * u], vr[d][2 * u + 1], scale);
#pragma unroll
                for (int r = 0; r < NR; ++r) oacc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r][u], oacc[r][d], 0, 0, 0);
            }
    };

    // A tile's K is on its way while the one before it is weighed, its V while its scores are made; its pages are looked up a tile
    // earlier still, and asked for before the codes of the tile in between (loads return in order).
    int t = t0 + wave;
    if (t < t1) {
        const Pages now = find(t);
        Pages at = find(min(t + NW, t1 - 1));
        load_k(t, now.k);
        load_v(t, now.v);
        for (; t < t1; t += NW) {
            const Pages then = find(min(t + 2 * NW, t1 - 1));
            scores();
            __builtin_amdgcn_sched_barrier(0);
            load_k(t + NW, at.k);
            __builtin_amdgcn_sched_barrier(0);
            softmax(t);
            weigh(t);
            __builtin_amdgcn_sched_barrier(0);
            load_v(t + NW, at.v);
            at = then;
        }
    }
    if (poisoned) {
        // once more through the tiles at an edge: a NaN for every row that sees a NaN code, in that code's column
        for (t = t0 + wave; t < t1; t += NW) {
            const int key0 = tile_of(t) * kTile, key = key0 + 16 * grp;
            load_v(t, lookup(key));
            if (!at_edge(key0, at_v)) continue;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const unsigned visible = sees(key, hi[r], lo[r], at_v >= 0);
                u32x4 see[2];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    see[j / 4][j % 4] = (visible >> (2 * j) & 1) * 0x3f80u | (visible >> (2 * j + 1) & 1) * 0x3f800000u;     // ones in bf16
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        u32x4 ind;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned nan = nan_codes(vr[d][2 * u + j / 2]) >> (16 * (j % 2) + 7);
                            ind[j] = (nan & 1) * 0x3f80u | (nan >> 8 & 1) * 0x3f800000u;
                        }
                        hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ind), __builtin_bit_cast(bf16x8, see[u]), hits, 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[r][d][e] = hits[e] > 0.f ? NAN : oacc[r][d][e];
                }
            }
        }
    }

    // merge the wavefronts: each scales its O to the maximum over all of them
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const float l = sum_over_groups(l_run[r]);
        if (grp == 0) { s_ml[0][wave][r * kBlock + col] = m_run[r]; s_ml[1][wave][r * kBlock + col] = l; }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = r * kBlock + col;
        float m = s_ml[0][0][row];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, s_ml[0][w][row]);
        const float f = m_run[r] == -INFINITY ? 0.f : exp2_hw((m_run[r] - m) * c);
        if (first + row < R)
#pragma unroll
            for (int d = 0; d < DT; ++d) *(f32x4*)(s_o + (wave * ROWS + row) * PITCH + 16 * d + 4 * grp) = oacc[r][d] * f;
    }
    if (tid < ROWS && first + tid < R) {
        const int row = first + tid, i = row / g, h = row - i * g;
        const size_t rowi = ((size_t)b * p.Hq + hk * g + h) * p.Sq + i;
        float m = s_ml[0][0][tid], l = 0.f;
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, s_ml[0][w][tid]);
#pragma unroll
        for (int w = 0; w < NW; ++w) l += s_ml[1][w][tid] * (s_ml[0][w][tid] == -INFINITY ? 0.f : exp2_hw((s_ml[0][w][tid] - m) * c));
        const bool none = l == 0.f || i >= seen.rows;
        s_inv[tid] = none ? 0.f : 1.f / l;
        if (alone) {
            if (p.lse) p.lse[rowi] = none ? -INFINITY : m * p.scale + logf(l);
        } else {
            *(f32x2*)(p.ml + 2 * (rowi * p.splits + split)) = f32x2{none ? -INFINITY : m, none ? 0.f : l};
        }
    }
    __syncthreads();
    constexpr int QPR = D / 4;
    for (int item = tid; item < ROWS * QPR; item += NW * 64) {
        const int rr = item / QPR, d = item % QPR * 4, row = first + rr;
        if (row >= R) break;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) v += *(const f32x4*)(s_o + (w * ROWS + rr) * PITCH + d);
        const int i = row / g, h = row - i * g;
        if (alone) {
            const float inv = s_inv[rr];
            u32x2 w2 = {0, 0};
            if (inv != 0.f) w2 = u32x2{pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv)};
            *(u32x2*)(p.o + b * p.o_sb + (hk * g + h) * p.o_sh + (long long)i * p.o_ss + d) = w2;
        } else {
            *(f32x4*)(p.part + ((((size_t)b * p.Hq + hk * g + h) * p.Sq + i) * p.splits + split) * D + d) = v;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// More packed rows than a few blocks: a wavefront owns 32 of them (the columns of v_mfma_f32_32x32x16_bf16), the wavefronts of
// a workgroup share tiles of 64 keys, which are decoded once, on the way from memory through registers into LDS: K as
// [64][D] and V^T as [D][64] bf16, two stages of each.  While tile t is worked on, tile t + 1 is decoded and written, tile
// t + 2 is on its way into registers and the page numbers of tile t + 3 are looked up; one barrier per tile.
//
// Row m of a 32-key block of S^T stands for key m with bits 2 and 3 exchanged: then the eight scores that a lane holds for a
// step of 16 keys are those of eight consecutive keys, one 16-byte piece of its row of V^T.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kTileRows = 32;
__device__ __forceinline__ constexpr int key_of_row(int m) { return (m & 0x13) | ((m >> 1) & 4) | ((m << 1) & 8); }
// Rows of K (2 D bytes) and of V^T (128 bytes) in pieces of 16 bytes, their places exchanged so that 16 consecutive rows' reads of
// one piece hit all banks once (rows of 128 bytes: two of them per turn of the banks).
template <int PIECES> __device__ __forceinline__ constexpr int piece_offset(int row, int piece) {
    return row * PIECES * 16 + ((piece ^ (PIECES == 16 ? row & 15 : (row >> 1) & 7)) << 4);
}

template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv_tiles(KvAttnParams p) {
    constexpr int KS = D / 16, DB = D / 32, KP = D / 8;
    constexpr int NC = D * kTile / 16 / (NW * 64);        // 16-code pieces per thread, tile and matrix
    constexpr int STAGE = 2 * kTile * D * 2;              // bytes of a K and a V tile
    constexpr int ROWS = NW * kTileRows;
    __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
    // by stage, the last tile: whose group of 16 keys has no page; whose V has a NaN, and which (for tiles at an edge only)
    __shared__ __attribute__((aligned(16))) int s_gone[2][4];
    __shared__ int s_nan[2];
    __shared__ __attribute__((aligned(8))) unsigned short s_bits[2][D][4];

    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nb = gridDim.x, per_xcd = nb >> 3, bid = blockIdx.x;
    int logical = bid < per_xcd * 8 ? (bid & 7) * per_xcd + (bid >> 3) : bid;
    const int rowblk = p.row_wgs - 1 - logical % p.row_wgs; logical /= p.row_wgs;       // (the last rows see the most keys)
    const int split = logical % p.splits; logical /= p.splits;
    const int B = p.B, b = logical % B, hk = logical / B;                // (an XCD gets heads, and so sequences of all lengths)

    const int g = p.Hq / p.c.Hkv, R = g * p.Sq, first = rowblk * ROWS;
    const Seen seen = seen_tiles(p, b, g, first, ROWS);
    const int per = part_tiles(p, seen, lane);
    const int t0 = split * per, t1 = min(seen.count, t0 + per);
    const bool alone = p.splits == 1;                     // the result itself, no part of it
    if (!alone && t0 >= t1) { no_part<ROWS>(p, b, hk, g, first, split); return; }

    // this lane's row; rows past the last one see what it does and are not stored
    const int row = min(first + wave * kTileRows + (lane & 31), R - 1), row_i = row / g, hq = hk * g + row - row_i * g;
    const int most_i = max(seen.rows - 1, 0);
    auto high_of = [&](int i) __attribute__((always_inline)) { return p.causal ? min(seen.pos0 + min(i, most_i), seen.n - 1) : seen.n - 1; };
    auto low_of = [&](int i) __attribute__((always_inline)) { return p.window ? (int)max((long long)seen.pos0 + min(i, most_i) - p.window + 1, 0LL) : 0; };
    const int hi = high_of(row_i), lo = low_of(row_i);
    // its wavefront's and its workgroup's first and last rows
    const int w_row0 = min(first + wave * kTileRows, R - 1) / g, w_row1 = min(first + wave * kTileRows + kTileRows - 1, R - 1) / g;
    const int w_hi = high_of(w_row1), w_lo = low_of(w_row0);
    const int g_hi = high_of(first / g), g_lo = low_of(min(first + ROWS - 1, R - 1) / g);

    // The order of the tiles: those that every row sees whole, a0 ... a1 - 1, then the first tokens', then the others.
    const int end = seen.first + seen.count - seen.sink_tiles;
    const int a0 = min(end, max(seen.first, (g_lo + kTile - 1) / kTile)), a1 = max(a0, min(end, (g_hi + 1) / kTile));
    const int whole = a1 - a0;
    auto tile_of = [&](int t) __attribute__((always_inline)) {
        const int x = t - whole, y = x - seen.sink_tiles + seen.first;
        const int z = x < seen.sink_tiles ? x : y < a0 ? y : y + whole;
        return t < whole ? a0 + t : z;
    };

    // A wavefront's pieces lie in one page each: K piece n is key k_key + 8 (D 64: 16) n, codes from 16 k_c on; V piece n the 16
    // keys of group v_grp, row v_row + 64 n.  So page numbers and addresses are scalars.
    constexpr int KPI = 1024 / D;                         // keys per load of a wavefront
    const int page = p.c.page, page_log2 = p.c.page_log2;
    const int k_first = wave * (kTile / NW), k_key = k_first + lane / (D / 16), k_c = lane % (D / 16);
    const int v_grp = wave & 3, v_row = (wave >> 2) * NC * 64 + lane;
    typedef const int __attribute__((address_space(4))) * ScalarInts;
    const ScalarInts table = (ScalarInts)(p.c.table + b * p.c.pitch);
    int at_k, at_v;                                       // the pages of the tile that is loaded next, -1: none
    u32x4 kr[NC], vr[NC];
    unsigned ke, ve;                                      // biased exponents
    bool gap;                                             // whether the loaded V piece has no page
    auto lookup = [&](int key) __attribute__((always_inline)) {
        const int at = table[min(key, seen.n - 1) >> page_log2];
        return key < seen.n && (unsigned)at < (unsigned)p.c.P ? at : -1;
    };
    auto find = [&](int t) __attribute__((always_inline)) {           // (behind the last tile: the last one again)
        const int key0 = tile_of(min(t, t1 - 1)) * kTile;
        at_k = lookup(key0 + k_first);
        at_v = lookup(key0 + 16 * v_grp);
    };
    const unsigned k_lane = lane / (D / 16) * D + 16 * k_c, v_lane = v_row * page;
    auto load = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(min(t, t1 - 1)) * kTile;
        const size_t unit_k = (size_t)max(at_k, 0) * p.c.Hkv + hk, unit_v = (size_t)max(at_v, 0) * p.c.Hkv + hk;
        const unsigned char* const k = p.c.k + (unit_k * page + ((key0 + k_first) & (page - 1))) * D;
        const unsigned char* const v = p.c.v + unit_v * page * D + ((key0 + 16 * v_grp) & (page - 1));
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            kr[n] = *(const u32x4*)(k + k_lane + n * KPI * D);
            vr[n] = *(const u32x4*)(v + v_lane + n * 64 * page);
        }
        ke = p.c.ke[unit_k];
        ve = p.c.ve[unit_v];
        gap = at_v < 0;
    };
    // What tile t, loaded, needs before it is decoded: zeros where the sequence holds nothing, a note of groups without a page.
    // At an edge NaN must not meet the probability 0 of a row that does not see it: zeros too, and a note.
    auto mend = [&](int t) __attribute__((always_inline)) {
        if (t < whole && !gap) return;
        const int key0 = tile_of(min(t, t1 - 1)) * kTile, left = gap ? 0 : seen.n - (key0 + 16 * v_grp);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            unsigned bits = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bytes = min(max(left - 4 * j, 0), 4);
                unsigned w = vr[n][j] & (bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1);
                const unsigned nan = nan_codes(w) >> 7;
                if (t >= whole) w &= ~(nan * 0xffu);
                bits |= (nan * 0x10204080u >> 28) << (4 * j);                         // bytes 0 ... 3 to bits 0 ... 3
                vr[n][j] = w;
            }
            if (t >= whole) {
                s_bits[t & 1][v_row + 64 * n][v_grp] = (unsigned short)bits;
                if (bits) s_nan[t & 1] = t;
            }
        }
        if (gap) s_gone[t & 1][v_grp] = t;
    };
    // Lane offsets into a stage; the pieces of a row are found by exchanging address bits.
    unsigned k_read = piece_offset<KP>(key_of_row(lane & 31), half), v_read = kTile * D * 2 + piece_offset<8>(lane & 31, half);
    unsigned k_write = piece_offset<KP>(k_key, 2 * k_c), v_write = kTile * D * 2 + piece_offset<8>(v_row, 2 * v_grp);
    auto put = [&](int t) __attribute__((always_inline)) {
        const unsigned st = (t & 1) * STAGE;
        const float ks = __uint_as_float(ke << 23), vs = __uint_as_float(ve << 23);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            // (K rows n KPI further on: for D = 128 their pieces' places differ in bit 3)
            const unsigned kw = (k_write ^ (KP == 16 && (n & 1) ? 128u : 0u)) + st + n * KPI * D * 2;
            *(bf16x8*)(smem + kw) = decode(kr[n][0], kr[n][1], ks);
            *(bf16x8*)(smem + (kw ^ 16)) = decode(kr[n][2], kr[n][3], ks);
            *(bf16x8*)(smem + (v_write + st + n * 64 * 128)) = decode(vr[n][0], vr[n][1], vs);
            *(bf16x8*)(smem + ((v_write + st + n * 64 * 128) ^ 16)) = decode(vr[n][2], vr[n][3], vs);
        }
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    bf16x8 qf[KS];
    {
        const __bf16* const q = p.q + b * p.q_sb + hq * p.q_sh + (long long)min(row_i, most_i) * p.q_ss + 8 * half;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *(const bf16x8*)(q + 16 * s);
    }
    f32x16 oacc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[i][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const float c = p.scale_log2;

    f32x16 sc[2];
    bf16x8 pf[4];
    auto scores = [&](int t) __attribute__((always_inline)) {
        const unsigned at = k_read + (t & 1) * STAGE;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 kf = *(const bf16x8*)(smem + (at ^ (s << 5)) + 32 * kb * D * 2);
                sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], sc[kb], 0, 0, 0);
            }
        }
    };
    auto softmax = [&]() __attribute__((always_inline)) {
        float mx = sc[0][0];
#pragma unroll
        for (int j = 1; j < 32; ++j) mx = fmaxf(mx, sc[j / 16][j % 16]);
        const float m_new = fmaxf(m_run, max_across_halves(mx));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2_hw((m_run - m_use) * c), mc = m_use * c;
        m_run = m_new;
        float sum = 0.f;
        unsigned pk[16];
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float p0 = exp2_hw(fmaf(sc[j / 16][j % 16], c, -mc)), p1 = exp2_hw(fmaf(sc[j / 16][j % 16 + 1], c, -mc));
            sum += p0 + p1;
            pk[j / 2] = pack_bf16x2(p0, p1);
        }
        l_run = l_run * alpha + sum;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) pf[kk] = __builtin_bit_cast(bf16x8, (u32x4{pk[4 * kk], pk[4 * kk + 1], pk[4 * kk + 2], pk[4 * kk + 3]}));
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0)
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[i][e] *= alpha;
    };
    auto weigh = [&](int t) __attribute__((always_inline)) {
        const unsigned at = v_read + (t & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const bf16x8 vf = *(const bf16x8*)(smem + (at ^ (kk << 5)) + 32 * i * 128);
                oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[kk], oacc[i], 0, 0, 0);
            }
    };
    // a NaN for every row that sees one
    auto poison = [&](int t, unsigned visible) __attribute__((always_inline)) {
        for (int d = 0; d < D; ++d) {
            const u32x2 bits = *(const u32x2*)s_bits[t & 1][d];
            const unsigned b0 = __builtin_amdgcn_readfirstlane(bits[0]) >> (8 * half), b1 = __builtin_amdgcn_readfirstlane(bits[1]) >> (8 * half);
            if (__builtin_amdgcn_readfirstlane(bits[0] | bits[1]) == 0) continue;
            unsigned mine = visible & ((b0 & 0xff) | (b0 >> 8 & 0xff00) | (b1 & 0xff) << 16 | (b1 >> 8 & 0xff00) << 16);
            mine |= __shfl_xor(mine, 32);
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[i][e] = mine != 0 && d == 32 * i + 8 * (e / 4) + 4 * half + e % 4 ? NAN : oacc[i][e];
        }
    };
    // which of the 32 keys of this lane's scores its row sees
    auto seen_keys = [&](int key0, unsigned there) __attribute__((always_inline)) {
        auto upto = [](int n) __attribute__((always_inline)) { return (1u << min(max(n, 0), 8)) - 1; };
        unsigned visible = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int key = key0 + 16 * x + 8 * half;
            const unsigned bits = upto(hi - key + 1) & (~upto(lo - key) | upto(p.sinks - key));
            visible |= (there >> x & 1 ? bits & 0xff : 0) << (8 * x);
        }
        return visible;
    };

    if (t0 < t1) {
        if (tid < 8) { s_nan[tid & 1] = -1; s_gone[tid & 1][tid >> 1] = -1; }
        find(t0); load(t0); find(t0 + 1);
        barrier();
        mend(t0); put(t0); load(t0 + 1); find(t0 + 2);
        barrier();
    }
    auto groups = [&](int t) __attribute__((always_inline)) {                // which groups of 16 keys have a page
        const i32x4 gone = *(const i32x4*)s_gone[t & 1];
        unsigned there = 15;
#pragma unroll
        for (int x = 0; x < 4; ++x) if (__builtin_amdgcn_readfirstlane(gone[x]) == t) there &= ~(1u << x);
        return there;
    };
    int t = t0;
    for (; t < min(t1, whole); ++t) {
        asm volatile("" : "+v"(k_read), "+v"(v_read), "+v"(k_write), "+v"(v_write));     // (offsets are cheaper to make again than to keep)
        if (groups(t) != 15) break;                                          // a page is missing: the general loop goes on
        mend(t + 1);
        scores(t);
        put(t + 1); load(t + 2); find(t + 3);
        softmax();
        weigh(t);
        barrier();
    }
    for (; t < t1; ++t) {
        asm volatile("" : "+v"(k_read), "+v"(v_read), "+v"(k_write), "+v"(v_write));
        const int key0 = tile_of(t) * kTile;
        const unsigned there = groups(t);
        mend(t + 1);
        put(t + 1); load(t + 2); find(t + 3);
        // nothing for this wavefront behind its last row's position, or in front of its first row's window
        if (key0 <= w_hi && (key0 + kTile > w_lo || key0 < p.sinks)) {
            scores(t);
            const unsigned visible = seen_keys(key0, there);
#pragma unroll
            for (int j = 0; j < 32; ++j) sc[j / 16][j % 16] = visible >> j & 1 ? sc[j / 16][j % 16] : -INFINITY;
            softmax();
            weigh(t);
            if (__builtin_amdgcn_readfirstlane(s_nan[t & 1]) == t) poison(t, visible);
        }
        barrier();
    }

    const float l = sum_across_halves(l_run);
    const int r = first + wave * kTileRows + (lane & 31);
    if (r >= R) return;
    const size_t rowi = ((size_t)b * p.Hq + hq) * p.Sq + row_i;
    const bool none = l == 0.f || row_i >= seen.rows;
    if (alone) {
        const float inv = none ? 0.f : 1.f / l;
        __bf16* const o = p.o + b * p.o_sb + hq * p.o_sh + (long long)row_i * p.o_ss;
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const u32x2 w = {pack_bf16x2(oacc[x][4 * y] * inv, oacc[x][4 * y + 1] * inv), pack_bf16x2(oacc[x][4 * y + 2] * inv, oacc[x][4 * y + 3] * inv)};
                *(u32x2*)(o + 32 * x + 8 * y + 4 * half) = none ? u32x2{0, 0} : w;
            }
        if (half == 0 && p.lse) p.lse[rowi] = none ? -INFINITY : m_run * p.scale + logf(l);
    } else {
        float* const o = p.part + (rowi * p.splits + split) * D;
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) *(f32x4*)(o + 32 * x + 8 * y + 4 * half) = f32x4{oacc[x][4 * y], oacc[x][4 * y + 1], oacc[x][4 * y + 2], oacc[x][4 * y + 3]};
        if (half == 0) *(f32x2*)(p.ml + 2 * (rowi * p.splits + split)) = f32x2{none ? -INFINITY : m_run, none ? 0.f : l};
    }
}

// O and LSE of a row from the parts of its splits: one workgroup per row, D / 4 threads for a part, its loads in batches of NL in
// flight per thread (the parts come from L2 or the memory-side cache: latency counts).
template <int D>
__global__ __launch_bounds__(256) void attn_kv_combine(KvAttnParams p) {
    constexpr int QPR = D / 4, NS = 256 / QPR, NL = 8, NM = kMaxKvSplits / 64;
    __shared__ float s_red[NS][D];
    const int tid = threadIdx.x, lane = tid & 63, sl = tid / QPR, d = tid % QPR * 4, S = p.splits;
    const unsigned rowi = blockIdx.x, bh = rowi / (unsigned)p.Sq;
    const int i = rowi - bh * p.Sq, b = bh / (unsigned)p.Hq, hq = bh - b * p.Hq;
    const float* const part = p.part + (size_t)rowi * S * D + d;
    const float* const ml = p.ml + 2 * ((size_t)rowi * S);
    f32x4 v[NL];
    auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int s = s0 + sl + n * NS;
            v[n] = s < S ? *(const f32x4*)(part + (size_t)s * D) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    // the parts' weights: of part 64 j + lane in w[j]
    float mm[NM], ll[NM], w[NM], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < NM; ++j) {
        const int s = 64 * j + lane;
        const f32x2 x = s < S ? *(const f32x2*)(ml + 2 * s) : f32x2{-INFINITY, 0.f};
        mm[j] = x[0]; ll[j] = x[1];
    }
    load(0);
#pragma unroll
    for (int j = 0; j < NM; ++j) m = fmaxf(m, mm[j]);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
#pragma unroll
    for (int j = 0; j < NM; ++j) {
        w[j] = mm[j] == -INFINITY ? 0.f : exp2_hw((mm[j] - m) * p.scale_log2);
        l += ll[j] * w[j];
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kMaxKvSplits / (NL * NS); ++j) {
        if (j * NL * NS < S) {
            if (j > 0) load(j * NL * NS);
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                const int s = j * NL * NS + n * NS + sl;                              // (its weight's register does not depend on sl)
                const float ws = __shfl(w[(j * NL * NS + n * NS) / 64], s & 63), ms = __shfl(mm[(j * NL * NS + n * NS) / 64], s & 63);
                if (ms != -INFINITY) acc += v[n] * ws;                                // (a part without keys is not written)
            }
        }
    }
    *(f32x4*)&s_red[sl][d] = acc;
    __syncthreads();
    if (tid < D / 2) {
        float a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) { a0 += s_red[n][2 * tid]; a1 += s_red[n][2 * tid + 1]; }
        const bool none = l == 0.f;
        const float inv = none ? 0.f : 1.f / l;
        *(unsigned*)(p.o + b * p.o_sb + hq * p.o_sh + (long long)i * p.o_ss + 2 * tid) = none ? 0u : pack_bf16x2(a0 * inv, a1 * inv);
        if (tid == 0 && p.lse) p.lse[rowi] = none ? -INFINITY : m * p.scale + logf(l);
    }
}

}  // namespace

// Rows per workgroup: 16 where that is all there is, else 32 rows per wavefront that share decoded tiles.
KvAttnPlan attn_kv_plan(int B, int Hq, int Hkv, int Sq, int keys, int D, int splits) {
    KvAttnPlan plan;
    const long long R = (long long)(Hq / Hkv) * Sq;
    plan.rows = R <= kBlock ? kBlock : 4 * kTileRows;
    plan.waves = plan.rows == kBlock && (long long)B * Hkv < 512 ? 8 : 4;
    plan.row_wgs = (int)((R + plan.rows - 1) / plan.rows);
    plan.splits = splits;
    plan.keys = keys;
    if (splits == 0) {
        const int tiles = (keys + kTile - 1) / kTile, most = plan.rows == kBlock ? (tiles + plan.waves - 1) / plan.waves : (tiles + 3) / 4;
        const long long base = (long long)B * Hkv * plan.row_wgs;
        long long s = (plan.rows == kBlock ? 512 : 512) / base;
        if (s > most) s = most;
        plan.splits = s < 1 ? 1 : s > kMaxKvSplits ? kMaxKvSplits : (int)s;
    }
    (void)D;
    return plan;
}

template <int D>
static void launch(const KvAttnParams& p, const KvAttnPlan& plan, unsigned blocks, hipStream_t stream) {
    if (plan.rows == kBlock && plan.waves == 8) hipLaunchKernelGGL((attn_kv_rows<D, 1, 8>), dim3(blocks), dim3(512), 0, stream, p);
    else if (plan.rows == kBlock) hipLaunchKernelGGL((attn_kv_rows<D, 1, 4>), dim3(blocks), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((attn_kv_tiles<D, 4>), dim3(blocks), dim3(256), 0, stream, p);
}

int attn_kv_launch(KvAttnParams p, const KvAttnPlan& plan, hipStream_t stream) {
    p.row_wgs = plan.row_wgs; p.splits = plan.splits;
    p.most_tiles = (plan.keys + kTile - 1) / kTile;
    const double blocks = (double)p.B * p.c.Hkv * p.row_wgs * p.splits;
    if (blocks * 512 >= 4294967296.0) return -2;
    if (p.c.D == 128) launch<128>(p, plan, (unsigned)blocks, stream);
    else launch<64>(p, plan, (unsigned)blocks, stream);
    if (hipGetLastError() != hipSuccess) return -1;
    if (p.splits > 1) {
        const unsigned rows = (unsigned)p.B * p.Hq * p.Sq;
        if (p.c.D == 128) hipLaunchKernelGGL(attn_kv_combine<128>, dim3(rows), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL(attn_kv_combine<64>, dim3(rows), dim3(256), 0, stream, p);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}
