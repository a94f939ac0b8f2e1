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
//     scale and the page's address are per lane.  The probabilities are rounded to bf16, which the matrix instruction wants of
//     both operands; their sum is that of the unrounded ones.
// The keys are cut over the wavefronts of a workgroup and over `splits` workgroups; the wavefronts are merged through LDS,
// the workgroups of a row by attn_kv_join or attn_kv_combine from fp32 parts.
// What bounds it: reading the codes, or latency.  32 sequences of up to 8191 keys, 8 kv heads of 128: 63 us = 4.4 TB/s; 16 of up to
// 20000 keys with a window of 4096, 16 heads of 64: 25 us = 5.0 TB/s (a copy reaches 4.9); one of 131071 keys, one kv head: 13.6 us
// (10 and 3.5 in the two kernels); one of 2000 keys, 8 kv heads: 9.5 us (5.5 and 4).  Many rows have a kernel of their own below.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "kv_launch.h"

namespace {

using namespace gfx950;

constexpr int kTile = 64;            // keys per tile
constexpr int kBlock = 16;           // packed query rows per block
// The reference that scores are taken relative to is a maximum that a row had once: it is made anew only where a score exceeds it
// by more than this, as a power of two of the probability.  Neither fp32 sums nor bf16 probabilities lose anything by such a
// factor, and a tile is spared the exchange of its maximum between lanes and the rescaling.
constexpr float kSlack = 10.f;
__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }      // (the reference of a row that has seen nothing)

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
// Those that do not stand for a number in bf16, given the biased exponent: with the largest one that is written, 2^120, codes from
// 0x78 on, which are 256 and more, are infinities too.
__device__ __forceinline__ unsigned no_numbers(unsigned w, unsigned exponent) {
    return ((w & 0x7f7f7f7fu) + (exponent == 247 ? 0x08080808u : 0x01010101u)) & 0x80808080u;
}
// Of these, those that make a sum infinite upwards (without their sign) or downwards; NaN does both.
__device__ __forceinline__ unsigned upwards(unsigned w, unsigned odd) { return odd & (~w | nan_codes(w)); }
__device__ __forceinline__ unsigned downwards(unsigned w, unsigned odd) { return odd & (w | nan_codes(w)); }

// A part without keys: its rows' maxima say so, its O stays unwritten.
template <int ROWS>
__device__ __forceinline__ void no_part(const KvAttnParams& p, int b, int hk, int g, int first, int split) {
    const int row = first + (int)threadIdx.x, i = row / g, h = row - i * g;
    if (threadIdx.x < ROWS && i < p.Sq)
        *(f32x2*)(p.ml + 2 * ((((size_t)b * p.Hq + hk * g + h) * p.Sq + i) * p.splits + split)) = f32x2{-INFINITY, 0.f};
}

template <int D> constexpr int merge_pitch() { return D + 4; }      // floats per O row in the merge area

// One block of packed rows per workgroup, every wavefront all of it.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv_rows(KvAttnParams p) {
    constexpr int KC = D / 64;                 // 16-byte loads per key and lane
    constexpr int DT = D / 16;                 // 16-row blocks of O^T
    constexpr int PITCH = merge_pitch<D>();
    constexpr int ROWS = kBlock;

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

    // this lane's row: what it sees, and Q.  Rows past the last one see what the last one does and are not stored.
    bf16x8 qf[KC * 2];
    const int row = min(first + col, R - 1), i = min(row / g, max(seen.rows - 1, 0)), h = row - row / g * g;
    const int pos = seen.pos0 + i;
    const int hi = p.causal ? min(pos, seen.n - 1) : seen.n - 1;
    const int lo = p.window ? (int)max((long long)pos - p.window + 1, 0LL) : 0;
    int hi_all = hi, lo_all = lo;                            // what any row of the workgroup sees
    const __bf16* const q = p.q + b * p.q_sb + (hk * g + h) * p.q_sh + (long long)(row / g) * p.q_ss;      // (not i: no wait for the lengths)
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) qf[2 * c + u] = *(const bf16x8*)(q + (grp + 4 * c) * 16 + 8 * u);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) { hi_all = max(hi_all, __shfl_xor(hi_all, x)); lo_all = min(lo_all, __shfl_xor(lo_all, x)); }

    f32x4 oacc[DT];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = p.scale_log2, slack = kSlack / c;
    const int page = p.c.page, sub_k = col >> 2, key_k = col & 3;
    const int* const table = p.c.table + b * p.c.pitch;
    bool poisoned = false;                                   // NaN or infinities were met where only some rows see them

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
        edge = edge || key0 + kTile - 1 > hi || (key0 < lo && key0 + kTile > p.sinks);
        return __builtin_amdgcn_ballot_w64(edge) != 0;
    };

    f32x4 sc[4];
    bf16x8 pf[2];
    auto scores = [&]() __attribute__((always_inline)) {
        const float scale = __uint_as_float(ke << 23);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            sc[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ch = 0; ch < KC; ++ch)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bf16x8 kf = decode(kr[kt][ch][2 * u], kr[kt][ch][2 * u + 1], scale);
                    sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * ch + u], sc[kt], 0, 0, 0);
                }
        }
    };
    auto softmax = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(t) * kTile;
        if (at_edge(key0, at_v)) {
            const int key = key0 + 16 * grp;                 // this lane's scores are those of 16 keys from here on
            const unsigned visible = sees(key, hi, lo, at_v >= 0);
#pragma unroll
            for (int j = 0; j < 16; ++j) sc[j / 4][j % 4] = visible >> j & 1 ? sc[j / 4][j % 4] : -INFINITY;
        }
        float mx = sc[0][0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = fmaxf(mx, sc[j / 4][j % 4]);
        if (__builtin_amdgcn_ballot_w64(!(mx <= m_run + slack)) != 0) {
            const float m_new = fmaxf(m_run, max_over_groups(mx));
            const float alpha = exp2_hw((m_run - finite(m_new)) * c);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d) oacc[d] *= alpha;
        }
        const float mc = finite(m_run) * c;
        float sum = 0.f;
        unsigned pk[8];
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float p0 = exp2_hw(fmaf(sc[j / 4][j % 4], c, -mc)), p1 = exp2_hw(fmaf(sc[j / 4][j % 4 + 1], c, -mc));
            sum += p0 + p1;
            pk[j / 2] = pack_bf16x2(p0, p1);
        }
        l_run += sum;
        pf[0] = __builtin_bit_cast(bf16x8, (u32x4{pk[0], pk[1], pk[2], pk[3]}));
        pf[1] = __builtin_bit_cast(bf16x8, (u32x4{pk[4], pk[5], pk[6], pk[7]}));
    };
    auto weigh = [&](int t) __attribute__((always_inline)) {
        const int key0 = tile_of(t) * kTile;
        float scale = __uint_as_float(ve << 23);
        if (at_edge(key0, at_v)) {
            // Keys without a page have zeros: what was loaded for them are page 0's codes and exponent, which may stand for anything.
            // NaN and infinities become zero: the probability 0 of a row that does not see them must not meet them.
            const unsigned there = at_v >= 0 ? ~0u : 0u;
            scale = at_v >= 0 ? scale : 1.f;
            unsigned any = 0;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    vr[d][j] &= there;
                    any |= no_numbers(vr[d][j], ve);
                }
            if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
                const unsigned some = sees(key0 + 16 * grp, hi_all, lo_all, at_v >= 0);
                unsigned bad = 0;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned odd = no_numbers(vr[d][j], ve) >> 7;
                        vr[d][j] &= ~(odd * 0xffu);
                        bad |= (odd * 0x10204080u >> 28) << (4 * j);                  // bytes 0 ... 3 to bits 0 ... 3
                    }
                poisoned = poisoned || __builtin_amdgcn_ballot_w64((bad & some) != 0) != 0;
            }
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 vf = decode(vr[d][2 * u], vr[d][2 * u + 1], scale);
                oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u], oacc[d], 0, 0, 0);
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
        // once more through the tiles at an edge: what the rows that see NaN or an infinity get, in its column
        for (t = t0 + wave; t < t1; t += NW) {
            const int key0 = tile_of(t) * kTile, key = key0 + 16 * grp;
            load_v(t, lookup(key));
            if (!at_edge(key0, at_v)) continue;
            const unsigned visible = sees(key, hi, lo, at_v >= 0);
            auto ones = [](unsigned bits) __attribute__((always_inline)) { return (bits & 1) * 0x3f80u | (bits >> 8 & 1) * 0x3f800000u; };      // in bf16
            u32x4 see[2];
#pragma unroll
            for (int j = 0; j < 8; ++j) see[j / 4][j % 4] = ones((visible >> (2 * j) & 1) | (visible >> (2 * j + 1) & 1) << 8);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                f32x4 up = {0.f, 0.f, 0.f, 0.f}, down = {0.f, 0.f, 0.f, 0.f};         // how many a row sees
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    u32x4 ind[2];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned w = vr[d][2 * u + j / 2], odd = no_numbers(w, ve);
                        ind[0][j] = ones(upwards(w, odd) >> (16 * (j % 2) + 7));
                        ind[1][j] = ones(downwards(w, odd) >> (16 * (j % 2) + 7));
                    }
                    up = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ind[0]), __builtin_bit_cast(bf16x8, see[u]), up, 0, 0, 0);
                    down = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ind[1]), __builtin_bit_cast(bf16x8, see[u]), down, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (up[e] > 0.f) oacc[d][e] += INFINITY;
                    if (down[e] > 0.f) oacc[d][e] -= INFINITY;
                }
            }
        }
    }

    // merge the wavefronts: each scales its O to the maximum over all of them
    const float l = sum_over_groups(l_run);
    if (grp == 0) { s_ml[0][wave][col] = m_run; s_ml[1][wave][col] = l; }
    __syncthreads();
    float m = s_ml[0][0][col];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, s_ml[0][w][col]);
    const float f = m_run == -INFINITY ? 0.f : exp2_hw((m_run - m) * c);
    if (first + col < R)
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4*)(s_o + (wave * ROWS + col) * PITCH + 16 * d + 4 * grp) = oacc[d] * f;
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
//
// What bounds it: 2 x 1000 rows of 32 heads of 128 against up to 16301 keys take 390 to 402 us, 955 to 985 TFLOP/s (a large matrix
// product 1366); the matrix units are busy 49 % of that, the vector units 50 %, LDS 37 %: the wavefronts' turns at them overlap in part.
// Two workgroups on a CU (three for D = 64, which its 169 registers just miss without being asked: 4 x 1500 rows against 8000 keys
// 238 -> 183 us) measured better than one of eight wavefronts; codes kept as they are in LDS and decoded at every read 554 us;
// a wavefront's priority raised around its matrix instructions 408 to 422; the first 32 keys' probabilities made while the other 32
// keys' scores are 406; 64 rows per wavefront, one wavefront per SIMD, 746; 256 rows per workgroup in two groups half a tile
// apart 454, though 477 for two sequences of equal length, which take 521 here (then against the power limit).
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kTileRows = 32, kTileWaves = 4;
__device__ __forceinline__ constexpr int key_of_row(int m) { return (m & 0x13) | ((m >> 1) & 4) | ((m << 1) & 8); }
// Rows of K (2 D bytes) and of V^T (128 bytes) in pieces of 16 bytes, their places exchanged so that 16 consecutive rows' reads of
// one piece hit all banks once (rows of 128 bytes: two of them per turn of the banks).
template <int PIECES> __device__ __forceinline__ constexpr int piece_offset(int row, int piece) {
    return row * PIECES * 16 + ((piece ^ (PIECES == 16 ? row & 15 : (row >> 1) & 7)) << 4);
}

template <int D>
__global__ __launch_bounds__(kTileWaves * 64, D == 64 ? 3 : 2) void attn_kv_tiles(KvAttnParams p) {
    constexpr int KS = D / 16, DB = D / 32, KP = D / 8;
    constexpr int NC = D / 64;                            // 16-code pieces per thread, tile and matrix
    constexpr int STAGE = 2 * kTile * D * 2;              // bytes of a K and a V tile
    constexpr int ROWS = kTileWaves * kTileRows;
    __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
    // by stage and group of 16 keys, the last tile where the group has no page; where its V has NaN or infinities, and which codes go
    // upwards and downwards (for tiles at an edge only)
    __shared__ __attribute__((aligned(16))) int s_gone[2][4], s_odd[2][4];
    __shared__ __attribute__((aligned(8))) unsigned short s_bits[2][2][D][4];

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

    // Wavefront w decodes the 16 keys of group w, which lie in one page: the page's number, addresses and exponents are scalars.  K
    // piece n is key 16 w + k_row + 8 n (D = 128), codes from 16 k_c on; V piece n the 16 keys of row v_row + 64 n.
    // (Which lane has which piece: eight lanes side by side write to eight different places of 16 bytes modulo 128.)
    constexpr int KPI = 1024 / D;                         // keys per load of a wavefront
    const int page = p.c.page, page_log2 = p.c.page_log2;
    const int k_c = D == 128 ? (lane & 3) | (lane >> 1 & 4) : lane & 3;
    const int k_row = D == 128 ? (lane >> 2 & 1) | (lane >> 3 & 6) : (lane >> 1 & 2) | (lane >> 3 & 1) | (lane >> 2 & 12);
    const int v_row = lane << 1 & 14 | (lane >> 3 & 1) | (lane & 48);
    typedef const unsigned __attribute__((address_space(4))) * ScalarWords;
    const ScalarWords table = (ScalarWords)(p.c.table + b * p.c.pitch);
    const unsigned page_bytes = page * D;
    const int last_slot = (seen.n - 1) >> page_log2;
    int key;                                              // the first key of the group, in the tile that is loaded next,
    unsigned entry;                                       // and its table entry
    u32x4 kr[NC], vr[NC];
    unsigned ke, ve, shifts;                              // words with the loaded tile's biased exponents, and where in them
    bool gap;                                             // whether the loaded group has no page
    auto find = [&](int t) __attribute__((always_inline)) {           // (behind the last tile: the last one again)
        key = tile_of(min(t, t1 - 1)) * kTile + 16 * wave;
        entry = table[min(key >> page_log2, last_slot)];
    };
    const unsigned k_lane = k_row * D + 16 * k_c, v_lane = v_row * page;
    // (The exponents come by scalar loads: those are counted apart from the codes' loads, so that none of these is waited for early.
    // A byte's aligned word lies in the byte's own allocation, whatever its neighbours are.)
    auto load = [&]() __attribute__((always_inline)) {
        gap = !((int)(key < seen.n) & (int)(entry < (unsigned)p.c.P));
        const unsigned unit = (gap ? 0u : entry) * p.c.Hkv + hk;
        const unsigned long long at = (unsigned long long)unit * page_bytes;
        const unsigned char* const k = p.c.k + at + (key & (page - 1)) * D;
        const unsigned char* const v = p.c.v + at + (key & (page - 1));
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            kr[n] = *(const u32x4*)(k + k_lane + n * KPI * D);
            vr[n] = *(const u32x4*)(v + v_lane + n * 64 * page);
        }
        const unsigned long long ea = (unsigned long long)(p.c.ke + unit), va = (unsigned long long)(p.c.ve + unit);
        ke = *(ScalarWords)(ea & ~3ull);
        ve = *(ScalarWords)(va & ~3ull);
        shifts = (unsigned)(ea & 3) | (unsigned)(va & 3) << 8;
    };
    // What tile t, loaded, needs before it is decoded: zeros where the sequence holds nothing, a note of groups without a page (for
    // which page 0 was loaded: its exponents, which may be any byte, do not count).
    // At an edge NaN and infinities must not meet the probability 0 of a row that does not see them: zeros too, and a note.
    auto mend = [&](int t) __attribute__((always_inline)) {
        if (__builtin_expect(t < whole && !gap, 1)) return;
        const int left = gap ? 0 : seen.n - (tile_of(min(t, t1 - 1)) * kTile + 16 * wave);
        const unsigned exponent = ve >> (8 * (shifts >> 8)) & 0xff;
        unsigned any = 0;
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bytes = min(max(left - 4 * j, 0), 4);
                vr[n][j] &= bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1;
                any |= no_numbers(vr[n][j], exponent);
            }
        if (t >= whole && __builtin_expect(__builtin_amdgcn_ballot_w64(any != 0) != 0, 0)) {
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                unsigned up = 0, down = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned w = vr[n][j], odd = no_numbers(w, exponent);
                    up |= ((upwards(w, odd) >> 7) * 0x10204080u >> 28) << (4 * j);    // bytes 0 ... 3 to bits 0 ... 3
                    down |= ((downwards(w, odd) >> 7) * 0x10204080u >> 28) << (4 * j);
                    vr[n][j] &= ~((odd >> 7) * 0xffu);
                }
                s_bits[t & 1][0][v_row + 64 * n][wave] = (unsigned short)up;
                s_bits[t & 1][1][v_row + 64 * n][wave] = (unsigned short)down;
            }
            s_odd[t & 1][wave] = t;
        }
        if (gap) {
            s_gone[t & 1][wave] = t;
            ke = ve = 0x7f7f7f7f;
        }
    };
    // Lane offsets into a stage; the pieces of a row are found by exchanging address bits.
    unsigned k_read = piece_offset<KP>(key_of_row(lane & 31), half), v_read = kTile * D * 2 + piece_offset<8>(lane & 31, half);
    unsigned k_write = piece_offset<KP>(16 * wave + k_row, 2 * k_c), v_write = kTile * D * 2 + piece_offset<8>(v_row, 2 * wave);
    auto put = [&](int t) __attribute__((always_inline)) {
        const unsigned st = (t & 1) * STAGE;
        const float ks = __uint_as_float((ke >> (8 * (shifts & 3)) & 0xff) << 23), vs = __uint_as_float((ve >> (8 * (shifts >> 8)) & 0xff) << 23);
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
    const float c = p.scale_log2, slack = kSlack / c;

    f32x16 sc[2];
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
    // what is under way moves on by a tile
    auto advance = [&](int t) __attribute__((always_inline)) { put(t + 1); load(); find(t + 3); };
    // The probabilities of the two blocks of 32 keys, and O += V^T P^T: the second block's probabilities are made between the
    // first one's matrix instructions.
    auto weigh = [&](int t) __attribute__((always_inline)) {
        float mx = sc[0][0];
#pragma unroll
        for (int j = 1; j < 32; ++j) mx = fmaxf(mx, sc[j / 16][j % 16]);
        if (__builtin_amdgcn_ballot_w64(!(mx <= m_run + slack)) != 0) {
            const float m_new = fmaxf(m_run, max_across_halves(mx));
            const float alpha = exp2_hw((m_run - finite(m_new)) * c);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[i][e] *= alpha;
        }
        const float mc = finite(m_run) * c;
        const unsigned at = v_read + (t & 1) * STAGE;
        auto v_piece = [&](int kk, int i) __attribute__((always_inline)) { return *(const bf16x8*)(smem + (at ^ (kk << 5)) + 32 * i * 128); };
        unsigned pk[16];
        auto two = [&](int j) __attribute__((always_inline)) {                // probabilities 2 j and 2 j + 1
            const float p0 = exp2_hw(fmaf(sc[j / 8][2 * j % 16], c, -mc)), p1 = exp2_hw(fmaf(sc[j / 8][2 * j % 16 + 1], c, -mc));
            l_run += p0 + p1;
            pk[j] = pack_bf16x2(p0, p1);
        };
        auto p_piece = [&](int kk) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, (u32x4{pk[4 * kk], pk[4 * kk + 1], pk[4 * kk + 2], pk[4 * kk + 3]})); };
        bf16x8 vf[2][DB];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < DB; ++i) vf[kk][i] = v_piece(kk, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) two(j);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[kk][i], p_piece(kk), oacc[i], 0, 0, 0);
                vf[kk][i] = v_piece(kk + 2, i);
#pragma unroll
                for (int j = 0; j < 4 / DB; ++j) two(8 + (kk * DB + i) * (4 / DB) + j);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < DB; ++i) oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[kk][i], p_piece(kk + 2), oacc[i], 0, 0, 0);
    };
    // what the rows that see NaN or an infinity get, in its column
    auto poison = [&](int t, unsigned visible, unsigned odd) __attribute__((always_inline)) {
        const unsigned noted0 = (odd & 1) * 0xffffu | (odd >> 1 & 1) * 0xffff0000u, noted1 = (odd >> 2 & 1) * 0xffffu | (odd >> 3) * 0xffff0000u;
        for (int x = 0; x < 2 * D; ++x) {
            const int way = x / D, d = x % D;
            const u32x2 bits = *(const u32x2*)s_bits[t & 1][way][d];
            const unsigned w0 = __builtin_amdgcn_readfirstlane(bits[0]) & noted0, w1 = __builtin_amdgcn_readfirstlane(bits[1]) & noted1;
            if ((w0 | w1) == 0) continue;
            const unsigned b0 = w0 >> (8 * half), b1 = w1 >> (8 * half);
            unsigned mine = visible & ((b0 & 0xff) | (b0 >> 8 & 0xff00) | (b1 & 0xff) << 16 | (b1 >> 8 & 0xff00) << 16);
            mine |= __shfl_xor(mine, 32);
            const float far = way ? -INFINITY : INFINITY;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[i][e] += mine != 0 && d == 32 * i + 8 * (e / 4) + 4 * half + e % 4 ? far : 0.f;
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
        if (tid < 8) s_odd[tid & 1][tid >> 1] = s_gone[tid & 1][tid >> 1] = -1;
        find(t0); load(); find(t0 + 1);
        barrier();
        mend(t0); put(t0); load(); find(t0 + 2);
        barrier();
    }
    auto noted = [&](const int (&s)[2][4], int t) __attribute__((always_inline)) {      // for which groups of 16 keys
        return (unsigned)__builtin_amdgcn_ballot_w64(lane < 4 && s[t & 1][lane & 3] == t);
    };
    int t = t0;
    for (; t < min(t1, whole); ++t) {
        asm volatile("" : "+v"(k_read), "+v"(v_read), "+v"(k_write), "+v"(v_write));     // (offsets are cheaper to make again than to keep)
        if (noted(s_gone, t) != 0) break;                                        // a page is missing: the general loop goes on
        mend(t + 1);
        scores(t);
        advance(t);
        weigh(t);
        barrier();
    }
    for (; t < t1; ++t) {
        asm volatile("" : "+v"(k_read), "+v"(v_read), "+v"(k_write), "+v"(v_write));
        const int key0 = tile_of(t) * kTile;
        const unsigned there = ~noted(s_gone, t) & 15;
        mend(t + 1);
        advance(t);
        // nothing for this wavefront behind its last row's position, or in front of its first row's window
        if (key0 <= w_hi && (key0 + kTile > w_lo || key0 < p.sinks)) {
            scores(t);
            const unsigned visible = seen_keys(key0, there);
#pragma unroll
            for (int j = 0; j < 32; ++j) sc[j / 16][j % 16] = visible >> j & 1 ? sc[j / 16][j % 16] : -INFINITY;
            weigh(t);
            const unsigned odd = noted(s_odd, t);
            if (__builtin_expect(odd != 0, 0)) poison(t, visible, odd);
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

// O and LSE of a row from the parts of its splits: COLS columns of a row per workgroup, COLS / 4 threads for a part, its loads in
// batches of NL in flight per thread (the parts come from L2 or the memory-side cache: latency counts, and so one batch should do).
template <int D, int COLS>
__global__ __launch_bounds__(256) void attn_kv_combine(KvAttnParams p) {
    constexpr int QPR = COLS / 4, NS = 256 / QPR, NL = 8, NM = kMaxKvSplits / 64;
    __shared__ float s_red[NS][COLS];
    const int tid = threadIdx.x, lane = tid & 63, sl = tid / QPR, S = p.splits, col0 = blockIdx.y * COLS, d = tid % QPR * 4;
    const unsigned rowi = blockIdx.x, bh = rowi / (unsigned)p.Sq;
    const int i = rowi - bh * p.Sq, b = bh / (unsigned)p.Hq, hq = bh - b * p.Hq;
    const float* const part = p.part + (size_t)rowi * S * D + col0 + d;
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
    if (tid < COLS / 2) {
        float a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) { a0 += s_red[n][2 * tid]; a1 += s_red[n][2 * tid + 1]; }
        const bool none = l == 0.f;
        const float inv = none ? 0.f : 1.f / l;
        *(unsigned*)(p.o + b * p.o_sb + hq * p.o_sh + (long long)i * p.o_ss + col0 + 2 * tid) = none ? 0u : pack_bf16x2(a0 * inv, a1 * inv);
        if (tid == 0 && col0 == 0 && p.lse) p.lse[rowi] = none ? -INFINITY : m * p.scale + logf(l);
    }
}

// The same for up to kJoinParts parts: a wavefront per row, all its loads in flight at once, no LDS.  65536 rows of 4 parts,
// D = 128: 95 us by a workgroup per row, 29 so.
constexpr int kJoinParts = 16;
template <int D>
__global__ __launch_bounds__(256) void attn_kv_join(KvAttnParams p) {
    constexpr int QPR = D / 4, NS = 64 / QPR, NL = kJoinParts / NS;
    const int lane = threadIdx.x & 63, sl = lane / QPR, d = lane % QPR * 4, S = p.splits;
    const unsigned rowi = blockIdx.x * 4 + (threadIdx.x >> 6), bh = rowi / (unsigned)p.Sq;
    if (rowi >= (unsigned)p.B * p.Hq * p.Sq) return;
    const int i = rowi - bh * p.Sq, b = bh / (unsigned)p.Hq, hq = bh - b * p.Hq;
    const f32x2 ml = lane < S ? *(const f32x2*)(p.ml + 2 * ((size_t)rowi * S + lane)) : f32x2{-INFINITY, 0.f};
    f32x4 v[NL];
#pragma unroll
    for (int n = 0; n < NL; ++n) {
        const int s = n * NS + sl;
        v[n] = s < S ? *(const f32x4*)(p.part + ((size_t)rowi * S + s) * D + d) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float m = ml[0];
#pragma unroll
    for (int x = kJoinParts / 2; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    const float w = ml[0] == -INFINITY ? 0.f : exp2_hw((ml[0] - m) * p.scale_log2);
    float l = ml[1] * w;
#pragma unroll
    for (int x = kJoinParts / 2; x > 0; x >>= 1) l += __shfl_xor(l, x);
    m = __shfl(m, 0); l = __shfl(l, 0);                                               // (the lanes from kJoinParts on had no part)
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NL; ++n) {
        const float ws = __shfl(w, n * NS + sl), ms = __shfl(ml[0], n * NS + sl);
        if (ms != -INFINITY) acc += v[n] * ws;                                        // (a part without keys is not written)
    }
#pragma unroll
    for (int x = QPR; x < 64; x <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x);
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    const u32x2 out = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    if (sl == 0) *(u32x2*)(p.o + b * p.o_sb + hq * p.o_sh + (long long)i * p.o_ss + d) = none ? u32x2{0, 0} : out;
    if (lane == 0 && p.lse) p.lse[rowi] = none ? -INFINITY : m * p.scale + logf(l);
}

}  // namespace

// Time of a call in microseconds, from what was measured on shapes of 1 to 256 sequences, 1 to 64000 keys, 1 to 256 packed rows.
// A round of workgroups takes its start (lengths, page numbers, first codes) and end, and for its tiles the longer of what their
// arithmetic takes, which two workgroups of four wavefronts on a CU share, and of what HBM takes at 6.2 TB/s, or up to 1.4
// times that where both are alike.  Parts cost a second kernel and their traffic.
static double estimate(const KvAttnPlan& plan, long long pairs, long long rows, int tiles, int D) {
    const bool rows16 = plan.rows == kBlock, wide = D == 128, single = plan.waves == 1;
    const long long n = pairs * plan.row_wgs * plan.splits, slots = rows16 && plan.waves == 8 ? 256 : 256 * (wide ? 8 : 12) / plan.waves;      // on 256 CUs
    const double start = single ? 4.6 : rows16 ? (plan.waves == 8 ? (wide ? 6.6 : 5.6) : wide ? 5.2 : 4.8) : 6.5;
    // a step is a tile of every wavefront (rows) or of the workgroup: with one wavefront on a SIMD, with two, and with the CU full
    const double alone = single ? (wide ? 0.95 : 0.6) : rows16 ? (plan.waves == 8 ? (wide ? 2.5 : 1.0) : wide ? 1.3 : 0.72) : wide ? 1.21 : 0.95;
    const double full = single ? (wide ? 1.6 : 1.2) : rows16 ? (plan.waves == 8 ? alone : wide ? 2.1 : 1.6) : wide ? 2.07 : 1.87;
    const double two = rows16 || wide ? full : 1.33;
    const int per = (tiles + plan.splits - 1) / plan.splits, steps = rows16 ? (per + plan.waves - 1) / plan.waves : per;
    const double bytes = (double)tiles / plan.splits * kTile * D * 2 / plan.row_wgs;          // of a workgroup, its row blocks sharing an L2
    auto round = [&](long long wgs) {
        const double work = steps * (wgs * plan.waves <= 1024 ? alone : wgs * plan.waves <= 2048 ? two : full), hbm = wgs * bytes / 6.2e6;
        const double both = sqrt(work * work + hbm * hbm) * (rows16 && plan.waves == 8 ? 0.9 : 1.0);
        return start + (both > work ? (both > hbm ? both : hbm) : work);
    };
    double t = (double)(n / slots) * (n >= slots ? round(slots) : 0.0);
    if (n % slots) t += round(n % slots);
    if (plan.splits > 1) {
        const double each = rows * (plan.splits <= kJoinParts ? 0.00036 : 0.0014), parts = (double)rows * plan.splits * (D + 2) * 4 / 5.5e6;
        t += 4.0 + (each > parts ? each : parts) + 0.8 * parts;
    }
    return t;
}

// How many rows a workgroup takes, by how many wavefronts, and how the keys are cut: whatever is estimated to be the fastest.
// Measured, rows of 16 / of 128 per workgroup, sequences x keys, D = 128, 8 kv heads: 32 packed rows 1 x 64000 35.5 / 47.0 us,
// 64 x 1000 39.5 / 45.0; 64 rows 55.9 / 50.2, 61.1 / 46.6; 128 rows 96.6 / 57.4, but 1 x 1000 11.6 / 16.2.  A wavefront by itself
// or four, sequences x keys, 8 kv heads of 128: 256 x 60 10.4 / 22.4 us, 256 x 250 30.2 / 36.5, but 16 x 250 8.4 / 6.4; where several
// row blocks share keys that are cut it is slower than estimated (2 blocks, 1 x 3781 14.0 / 11.2), and left out.
KvAttnPlan attn_kv_plan(int B, int Hq, int Hkv, int Sq, int keys, int D, int splits, int wg_rows) {
    static const int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};
    const long long R = (long long)(Hq / Hkv) * Sq, pairs = (long long)B * Hkv, rows = (long long)B * Hq * Sq;
    const int tiles = (keys + kTile - 1) / kTile;
    KvAttnPlan best{};
    double least = 1e300;
    static const int kWaves[] = {8, 4, 1, kTileWaves};
    for (int kind = 0; kind < 4; ++kind) {
        KvAttnPlan plan;
        plan.rows = kind < 3 ? kBlock : kTileWaves * kTileRows;
        if (wg_rows ? plan.rows != wg_rows : kind < 3 && R > 512) continue;
        plan.waves = kWaves[kind];
        plan.row_wgs = (int)((R + plan.rows - 1) / plan.rows);
        plan.keys = keys;
        const int most = kind < 3 ? (tiles + plan.waves - 1) / plan.waves : (tiles + 1) / 2;
        for (int cut : kCuts) {
            if (splits == 0 && cut > 1 && cut > most) break;
            plan.splits = splits ? splits : cut;
            if (plan.waves == 1 && plan.splits > 1 && plan.row_wgs > 1) break;
            // (a given cut that is the library's own gets the shape that the library chose for it)
            const double t = estimate(plan, pairs, rows, tiles, D) + (plan.splits > 1 && plan.splits > most ? 1e9 : 0.0);
            if (t < least) { least = t; best = plan; }
            if (splits) break;
        }
    }
    return best;
}

template <int D>
static void launch(const KvAttnParams& p, const KvAttnPlan& plan, unsigned blocks, hipStream_t stream) {
    if (plan.rows == kBlock && plan.waves == 8) hipLaunchKernelGGL((attn_kv_rows<D, 8>), dim3(blocks), dim3(512), 0, stream, p);
    else if (plan.waves == 1) hipLaunchKernelGGL((attn_kv_rows<D, 1>), dim3(blocks), dim3(64), 0, stream, p);
    else if (plan.rows == kBlock) hipLaunchKernelGGL((attn_kv_rows<D, 4>), dim3(blocks), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(attn_kv_tiles<D>, dim3(blocks), dim3(kTileWaves * 64), 0, stream, p);
}

int attn_kv_launch(KvAttnParams p, const KvAttnPlan& plan, hipStream_t stream) {
    p.row_wgs = plan.row_wgs; p.splits = plan.splits;
    p.most_tiles = (plan.keys + kTile - 1) / kTile;
    const double blocks = (double)p.B * p.c.Hkv * p.row_wgs * p.splits;
    if (blocks * 512 >= 4294967296.0 || (p.splits > 1 && (double)p.B * p.Hq * p.Sq * 256 >= 4294967296.0)) return -2;
    if (p.c.D == 128) launch<128>(p, plan, (unsigned)blocks, stream);
    else launch<64>(p, plan, (unsigned)blocks, stream);
    if (hipGetLastError() != hipSuccess) return -1;
    if (p.splits > 1) {
        const unsigned rows = (unsigned)p.B * p.Hq * p.Sq;
        // 32 columns per workgroup where all of them would take more than one batch of loads: 8 rows of 256 parts, call 16.4 -> 13.9
        // us; 32 rows of 64 parts, one batch, 9.4 and 9.5
        const int D = p.c.D;
        if (p.splits <= kJoinParts) hipLaunchKernelGGL((D == 128 ? attn_kv_join<128> : attn_kv_join<64>), dim3((rows + 3) / 4), dim3(256), 0, stream, p);
        else if (p.splits > 8 * (256 / (D / 4))) hipLaunchKernelGGL((D == 128 ? attn_kv_combine<128, 32> : attn_kv_combine<64, 32>), dim3(rows, D / 32), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((D == 128 ? attn_kv_combine<128, 128> : attn_kv_combine<64, 64>), dim3(rows), dim3(256), 0, stream, p);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}
