// Writing the quantised cache and reading it back, for gfx950.  What bounds both: reading and writing every value once, or, for
// a token per sequence, a chain of latencies (lengths, page, exponent).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "kv_launch.h"

namespace {

using namespace gfx950;

constexpr int kThreads = 256;
constexpr int kLeastExp = -100;
constexpr int kReadRows = 64;        // positions per workgroup of kv_read

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }    // -126 <= e <= 127

// The least e >= kLeastExp with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_for(float amax) {
    const unsigned bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kLeastExp ? kLeastExp : e;
}

// Eight codes of x * f; NaN and infinities are 0x7f.  w: eight bf16 bit patterns in four dwords.
__device__ __forceinline__ u32x2 codes_of(u32x4 w, float f) {
    u32x2 out;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float x0 = __uint_as_float(w[2 * j] << 16), x1 = __uint_as_float(w[2 * j] & 0xffff0000u);
        const float x2 = __uint_as_float(w[2 * j + 1] << 16), x3 = __uint_as_float(w[2 * j + 1] & 0xffff0000u);
        unsigned c = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * f, x1 * f, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x2 * f, x3 * f, c, true);
        const unsigned odd = (fabsf(x0) < INFINITY ? 0u : 0xffu) | (fabsf(x1) < INFINITY ? 0u : 0xff00u) |
                             (fabsf(x2) < INFINITY ? 0u : 0xff0000u) | (fabsf(x3) < INFINITY ? 0u : 0xff000000u);
        out[j] = (c & ~odd) | (0x7f7f7f7fu & odd);
    }
    return out;
}
// Four codes rounded again to c * f; the NaN codes stay.
__device__ __forceinline__ unsigned again(unsigned w, float f) {
    const unsigned nan = ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    unsigned c = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, c, true);
    return (c & ~nan) | (w & nan);
}
// The largest finite |x| of eight values, as the bits of a bf16 (which order as the values do).
__device__ __forceinline__ unsigned largest(u32x4 w, unsigned m) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned lo = w[j] & 0x7fffu, hi = w[j] >> 16 & 0x7fffu;
        m = max(m, lo < 0x7f80u ? lo : 0u);
        m = max(m, hi < 0x7f80u ? hi : 0u);
    }
    return m;
}

// A unit is the keys or the values of one page and kv head, so that the page's exponent, its earlier tokens' codes and its new
// ones are one unit's business: a wavefront for pages of up to 32 tokens, 256 threads for larger ones.  A thread reads blocks of 4
// tokens x 8 values, once, keeps them while the page's maximum is found, and packs the codes of V by four tokens: the transposed
// page is put together in LDS and leaves in pieces of 16 tokens; pieces with other tokens too were read before, and leave whole.
// 4 prompts of up to 4096 tokens, 8 heads of 128, pages of 64: 14.8 us = 4.2 TB/s (37 us with a second pass over the values and
// single bytes of V).
// FEW: at most kFewTokens new tokens lie in few blocks and two pieces, for which a wavefront does on larger pages too: one token of
// 99 sequences and 16 heads, pages of 64, 15.8 -> 11.3 us, 16 of 16 sequences and 8 heads, pages of 128, 8.4 -> 7.1 (17 tokens, by 256
// threads, 8.6).  One token of 64 sequences, 8 heads, pages of 16 / 64 / 128: 5.3 / 6.9 / 7.4 us in a captured graph (every column's
// byte of V lies in another line); 7.4 / 12.0 / 15.8 between two events where scales grow, 7.0 / 8.7 / 9.4 where they do not.
constexpr int kFewTokens = 16;
template <int D, int PAGE, bool FEW>
__global__ __launch_bounds__(kThreads) void kv_write(KvWriteParams p) {
    constexpr int TPU = PAGE <= 32 || FEW ? 64 : 256, UNITS = kThreads / TPU;
    constexpr int QS = FEW ? kFewTokens / 4 + 1 : PAGE / 4, CPR = D / 8, BLOCKS = QS * CPR, NB = (BLOCKS + TPU - 1) / TPU;
    constexpr int PPR = FEW ? 2 : PAGE / 16, NP = D * PPR / TPU;       // pieces of 16 tokens of V per row d, and per thread
    constexpr int PITCH = QS | 1;                                      // dwords per row d in LDS
    __shared__ unsigned s_page[UNITS][D * PITCH];
    __shared__ unsigned s_max[kThreads / 64];
    const int tid = threadIdx.x % TPU, sub = UNITS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPU);
    const bool is_v = blockIdx.y != 0;
    unsigned id = blockIdx.x * UNITS + sub;
    const int h = id % (unsigned)p.c.Hkv; id /= (unsigned)p.c.Hkv;
    const int f = id % (unsigned)p.F, b = id / (unsigned)p.F;

    // the unit's tokens: `held` earlier ones of the page, then `fresh` new ones; none where there is nothing to do.  (The new values
    // are on their way before it is known whether the page is there: one latency less.)
    int held = 0, fresh = 0, at = -1;
    long long token0 = 0;                                              // of the new ones, the first
    if (b < p.B) {
        const long long start = p.start[b];
        const int n = p.count ? min(max(p.count[b], 0), p.S) : p.S;
        const long long pg = (start >> p.c.page_log2) + f;             // (arithmetic shift: rounds down)
        const long long base = pg << p.c.page_log2;                    // the page's first position
        const long long lo = start > base ? start : base, hi = start + n < base + PAGE ? start + n : base + PAGE;
        if (pg >= 0 && pg < p.c.W && lo < hi) {
            at = p.c.table[b * p.c.pitch + pg];
            held = (int)(lo - base); fresh = (int)(hi - lo); token0 = lo - start;
        }
    }
    const long long row = is_v ? p.v_ss : p.k_ss;
    const __bf16* const src = (is_v ? p.v + b * p.v_sb + h * p.v_sh : p.k + b * p.k_sb + h * p.k_sh) + (token0 - held) * row;   // of token 0 of the page

    const int q0 = FEW ? held / 4 : 0, p0 = FEW ? held / 16 : 0;       // the first block and piece
    u32x4 x[NB][4];
    unsigned m = 0;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int blk = n * TPU + tid, q = q0 + blk / CPR, c = blk % CPR;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = blk < BLOCKS ? 4 * q + j : PAGE;
            x[n][j] = u32x4{0, 0, 0, 0};
            if (t >= held && t < held + fresh) x[n][j] = *(const u32x4*)(src + t * row + c * 8);
        }
    }
    if (at < 0 || at >= p.c.P) fresh = 0;
    if (TPU == 256 && fresh == 0) return;
    const size_t unit = (size_t)(fresh ? at : 0) * p.c.Hkv + h;
    unsigned char* const codes = (is_v ? p.c.v : p.c.k) + unit * PAGE * D;
    unsigned char* const exps = (is_v ? p.c.ve : p.c.ke) + unit;
    int e_old = fresh ? (int)*exps - 127 : 0;
    // pieces of V that hold other tokens than new ones too
    u32x4 old[NP];
    auto piece_at = [&](int n, int& d) __attribute__((always_inline)) {
        const int i = n * TPU + tid;
        d = i / PPR;
        return 16 * (p0 + i % PPR);
    };
    auto mixed = [&](int t) __attribute__((always_inline)) { return t < held + fresh && t + 16 > held && (t < held || t + 16 > held + fresh); };
    if (is_v)
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            int d;
            const int t = piece_at(n, d);
            if (fresh > 0 && mixed(t)) old[n] = *(const u32x4*)(codes + d * PAGE + t);
        }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = largest(x[n][j], m);
#pragma unroll
    for (int y = 32; y > 0; y >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, y));
    if constexpr (TPU == 256) {
        if ((tid & 63) == 0) s_max[tid >> 6] = m;
        __syncthreads();                                               // (and every thread has read the old exponent)
        m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    }
    int e = exponent_for(__uint_as_float(m << 16));
    if (held > 0 && e < e_old) e = e_old;

    // a scale that has grown: the earlier tokens' codes are rounded again, those of V that lie in a piece with new ones further down
    const bool grown = held > 0 && fresh > 0 && e > e_old;
    const float f2 = grown ? two_to(max(e_old - e, -126)) : 1.f;
    if (grown) {
        const int first = held / 16, count = is_v ? D * first : held * (D / 16);
        for (int i = tid; i < count; i += TPU) {
            u32x4* const c = (u32x4*)(codes + (is_v ? i / first * PAGE + i % first * 16 : i * 16));
            *c = u32x4{again((*c)[0], f2), again((*c)[1], f2), again((*c)[2], f2), again((*c)[3], f2)};
        }
    }
    const float f1 = two_to(-e);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int blk = n * TPU + tid, q = q0 + blk / CPR, c = blk % CPR;
        if (BLOCKS % TPU != 0 && blk >= BLOCKS) break;
        if (4 * q + 4 <= held || 4 * q >= held + fresh) continue;      // (no new token: what lies in LDS there is not used)
        u32x2 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = codes_of(x[n][j], f1);
        if (!is_v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 4 * q + j;
                if (t >= held && t < held + fresh) *(u32x2*)(codes + t * D + c * 8) = w[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int s = 8 * (i % 4);
                s_page[sub][(c * 8 + i) * PITCH + q - q0] = (w[0][i / 4] >> s & 0xff) | (w[1][i / 4] >> s & 0xff) << 8 | (w[2][i / 4] >> s & 0xff) << 16 | (w[3][i / 4] >> s & 0xff) << 24;
            }
        }
    }
    if (is_v && fresh > 0) {
        if constexpr (TPU == 256) __syncthreads();
        else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (a wavefront reads what it wrote itself)
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            int d;
            const int t = piece_at(n, d);
            if (t >= held + fresh || t + 16 <= held) continue;
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = s_page[sub][d * PITCH + min(max(t / 4 + j - q0, 0), QS - 1)];
            if (mixed(t)) {                                            // earlier tokens, new ones, and what lies behind them
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    auto bytes = [](int n) __attribute__((always_inline)) { n = min(max(n, 0), 4); return n == 4 ? ~0u : (1u << (8 * n)) - 1; };
                    const unsigned was = bytes(held - t - 4 * j), now = bytes(held + fresh - t - 4 * j) & ~was;
                    w[j] = ((grown ? again(old[n][j], f2) : old[n][j]) & was) | (w[j] & now) | (old[n][j] & ~(was | now));
                }
            }
            *(u32x4*)(codes + d * PAGE + t) = w;
        }
    }
    if (tid == 0 && fresh > 0) *exps = (unsigned char)(e + 127);
}

// Sixteen codes as bf16, times scale: eight dwords of two.
__device__ __forceinline__ void decode16(u32x4 c, float scale, unsigned (&out)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        out[2 * j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[j], scale, false));
        out[2 * j + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[j], scale, true));
    }
}

// 64 positions of one sequence and kv head, keys (blockIdx.y 0) or values.  Keys go straight through; a thread with values holds
// 16 tokens of two columns, which meet their rows in LDS (dword c of the rows of group g lies at c ^ 16 g: no bank conflicts).
// 8 sequences of up to 4001 positions, 8 heads of 128: 34.5 us a call = 4.9 TB/s (25 in the kernel while the codes are still cached).
// From a position inside a group of 16 on, V goes code by code: 44 us in place of 26 in a captured graph.
template <int D>
__global__ __launch_bounds__(kThreads) void kv_read(KvReadParams p) {
    constexpr int CPR = D / 16, NK = kReadRows * CPR / kThreads;
    __shared__ __attribute__((aligned(16))) unsigned s_rows[kReadRows * D / 2];
    const int tid = threadIdx.x, page = p.c.page;
    const unsigned tiles = (unsigned)((p.S + kReadRows - 1) / kReadRows);
    unsigned id = blockIdx.x;
    const int s0 = (int)(id % tiles) * kReadRows; id /= tiles;
    const int h = id % (unsigned)p.c.Hkv, b = id / (unsigned)p.c.Hkv;
    const int n = p.lens[b];
    // a position's codes' page, -1 where there is none
    auto lookup = [&](long long pos) __attribute__((always_inline)) {
        if (pos >= n || (pos >> p.c.page_log2) >= p.c.W) return -1;
        const int at = p.c.table[b * p.c.pitch + (pos >> p.c.page_log2)];
        return at >= 0 && at < p.c.P ? at : -1;
    };
    if (blockIdx.y == 0) {
        __bf16* const out = p.k + b * p.k_sb + h * p.k_sh;
        u32x4 c[NK];
        float scale[NK];
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            const int i = x * kThreads + tid, s = s0 + i / CPR;
            const long long pos = (long long)p.first + s;
            const int at = s < p.S ? lookup(pos) : -1;
            c[x] = u32x4{0, 0, 0, 0};
            scale[x] = 1.f;
            if (at >= 0) {
                const size_t unit = (size_t)at * p.c.Hkv + h;
                c[x] = *(const u32x4*)(p.c.k + (unit * page + (pos & (page - 1))) * D + 16 * (i % CPR));
                scale[x] = __uint_as_float((unsigned)p.c.ke[unit] << 23);
            }
        }
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            const int i = x * kThreads + tid, s = s0 + i / CPR;
            unsigned w[8];
            decode16(c[x], scale[x], w);
            if (s < p.S) {
                u32x4* const o = (u32x4*)(out + s * p.k_ss + 16 * (i % CPR));
                o[0] = u32x4{w[0], w[1], w[2], w[3]};
                o[1] = u32x4{w[4], w[5], w[6], w[7]};
            }
        }
    } else {
        if (p.first % 16 == 0) {
            if (tid < 2 * D) {
                const int g = tid & 3, d = tid >> 2 << 1;              // (groups side by side: 64 consecutive codes of a column)
                const long long pos = (long long)p.first + s0 + 16 * g;
                const int at = lookup(pos);
                u32x4 c[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                float scale = 1.f;
                if (at >= 0) {
                    const size_t unit = (size_t)at * p.c.Hkv + h;
                    const unsigned char* const v = p.c.v + unit * page * D + (pos & (page - 1));
                    c[0] = *(const u32x4*)(v + d * page);
                    c[1] = *(const u32x4*)(v + d * page + page);
                    scale = __uint_as_float((unsigned)p.c.ve[unit] << 23);
                }
                unsigned w0[8], w1[8];
                decode16(c[0], scale, w0);
                decode16(c[1], scale, w1);
                const int left = (int)min((long long)n - pos, 16LL);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const unsigned s = 16 * (j % 2), pair = (w0[j / 2] >> s & 0xffff) | (w1[j / 2] >> s) << 16;
                    s_rows[(16 * g + j) * (D / 2) + (d / 2 ^ (16 * g & (D / 2 - 1)))] = j < left ? pair : 0u;
                }
            }
        } else {
            // a start inside a group of 16: code by code
            for (int i = tid; i < kReadRows * D / 2; i += kThreads) {
                const int t = i % kReadRows, d = i / kReadRows * 2;
                const long long pos = (long long)p.first + s0 + t;
                const int at = lookup(pos);
                unsigned pair = 0;
                if (at >= 0) {
                    const size_t unit = (size_t)at * p.c.Hkv + h;
                    const unsigned char* const v = p.c.v + unit * page * D + d * page + (pos & (page - 1));
                    pair = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)v[0] | (unsigned)v[page] << 8,
                                                                                                __uint_as_float((unsigned)p.c.ve[unit] << 23), false));
                }
                s_rows[t * (D / 2) + (d / 2 ^ (16 * (t / 16) & (D / 2 - 1)))] = pair;
            }
        }
        __syncthreads();
        __bf16* const out = p.v + b * p.v_sb + h * p.v_sh;
        for (int i = tid; i < kReadRows * (D / 8); i += kThreads) {
            const int t = i / (D / 8), c = i % (D / 8);
            if (s0 + t < p.S) *(u32x4*)(out + (s0 + t) * p.v_ss + 8 * c) = *(const u32x4*)&s_rows[t * (D / 2) + 4 * (c ^ (4 * (t / 16) & (D / 8 - 1)))];
        }
    }
}

// The same for at most kFewTokens positions, which lie in two groups of 16: keys (blockIdx.y 0) by pieces of 16 columns of rows one
// after the other, values by a wavefront per sequence and head whose lanes take two columns each.  Heads x sequences of 128 columns:
// one position of 8 x 6767, pages of 16, 121 -> 33 us; 8 of 8 x 3296 73 -> 34; 16 of 8 x 1000 23.1 -> 20.5 (17: 24); 16 of 8 x 16 3.3 and
// 3.7.  What a few positions cannot do without is a piece of a line of V for every column: three of 4 x 12540, pages of 64, 108 us.
template <int D>
__global__ __launch_bounds__(kThreads) void kv_read_few(KvReadParams p) {
    constexpr int CPR = D / 16, UNITS = kThreads / 64;
    __shared__ __attribute__((aligned(16))) unsigned s_rows[UNITS][kFewTokens * D / 2];
    const int page = p.c.page;
    auto lookup = [&](int b, int n, long long pos) __attribute__((always_inline)) {
        if (pos >= n || (pos >> p.c.page_log2) >= p.c.W) return -1;
        const int at = p.c.table[b * p.c.pitch + (pos >> p.c.page_log2)];
        return at >= 0 && at < p.c.P ? at : -1;
    };
    if (blockIdx.y == 0) {
        const unsigned id = blockIdx.x * kThreads + threadIdx.x, row = id / CPR, bh = row / (unsigned)p.S;
        const int c = id % CPR, s = row - bh * p.S, b = bh / (unsigned)p.c.Hkv, h = bh - b * p.c.Hkv;
        if (b >= p.B) return;
        const long long pos = (long long)p.first + s;
        const int at = lookup(b, p.lens[b], pos);
        u32x4 codes = {0, 0, 0, 0};
        float scale = 1.f;
        if (at >= 0) {
            const size_t unit = (size_t)at * p.c.Hkv + h;
            codes = *(const u32x4*)(p.c.k + (unit * page + (pos & (page - 1))) * D + 16 * c);
            scale = __uint_as_float((unsigned)p.c.ke[unit] << 23);
        }
        unsigned w[8];
        decode16(codes, scale, w);
        u32x4* const o = (u32x4*)(p.k + b * p.k_sb + h * p.k_sh + s * p.k_ss + 16 * c);
        o[0] = u32x4{w[0], w[1], w[2], w[3]};
        o[1] = u32x4{w[4], w[5], w[6], w[7]};
        return;
    }
    const int lane = threadIdx.x & 63, sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned id = blockIdx.x * UNITS + sub;
    const int b = (int)(id / (unsigned)p.c.Hkv), h = (int)(id % (unsigned)p.c.Hkv);
    if (b >= p.B) return;                                              // (no barrier below: a wavefront reads what it wrote itself)
    const int n = p.lens[b], skip = p.first & 15, d = 2 * lane;
    if (d < D)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            if (16 * g - skip >= p.S) break;
            const long long pos = (long long)p.first - skip + 16 * g;
            // (a group that begins before the first position is there if that position is)
            const int at = lookup(b, n, g == 0 ? (long long)p.first : pos);
            u32x4 c[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
            float scale = 1.f;
            if (at >= 0) {
                const size_t unit = (size_t)at * p.c.Hkv + h;
                const unsigned char* const v = p.c.v + unit * page * D + d * page + (pos & (page - 1));
                c[0] = *(const u32x4*)v;
                c[1] = *(const u32x4*)(v + page);
                scale = __uint_as_float((unsigned)p.c.ve[unit] << 23);
            }
            unsigned w0[8], w1[8];
            decode16(c[0], scale, w0);
            decode16(c[1], scale, w1);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int t = 16 * g + j - skip;
                const unsigned x = 16 * (j % 2), pair = (w0[j / 2] >> x & 0xffff) | (w1[j / 2] >> x) << 16;
                if (t >= 0 && t < p.S) s_rows[sub][t * (D / 2) + lane] = pos + j < n ? pair : 0u;
            }
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    __bf16* const out = p.v + b * p.v_sb + h * p.v_sh;
    for (int i = lane; i < p.S * (D / 8); i += 64) {
        const int t = i / (D / 8), c = i % (D / 8);
        *(u32x4*)(out + t * p.v_ss + 8 * c) = *(const u32x4*)&s_rows[sub][t * (D / 2) + 4 * c];
    }
}

}  // namespace

template <int PAGE, bool FEW>
static void launch_write(const KvWriteParams& p, dim3 grid, hipStream_t stream) {
    if (p.c.D == 128) hipLaunchKernelGGL((kv_write<128, PAGE, FEW>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((kv_write<64, PAGE, FEW>), grid, dim3(kThreads), 0, stream, p);
}

int kv_write_launch(const KvWriteParams& p, hipStream_t stream) {
    const double units = (double)p.B * p.F * p.c.Hkv;
    const bool few = p.c.page >= 64 && p.S <= kFewTokens;
    const int per = p.c.page <= 32 || few ? 4 : 1;
    const double blocks = (units + per - 1) / per;
    if (blocks * kThreads >= 4294967296.0) return -2;
    const dim3 grid((unsigned)blocks, 2);
    if (p.c.page == 16) launch_write<16, false>(p, grid, stream);
    else if (p.c.page == 32) launch_write<32, false>(p, grid, stream);
    else if (p.c.page == 64 && few) launch_write<64, true>(p, grid, stream);
    else if (p.c.page == 64) launch_write<64, false>(p, grid, stream);
    else if (few) launch_write<128, true>(p, grid, stream);
    else launch_write<128, false>(p, grid, stream);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int kv_read_launch(const KvReadParams& p, hipStream_t stream) {
    const bool few = p.S <= kFewTokens;
    const double units = (double)p.B * p.c.Hkv;
    const double blocks = few ? fmax(ceil(units * p.S * (p.c.D / 16) / kThreads), ceil(units / (kThreads / 64))) : units * ((p.S + kReadRows - 1) / kReadRows);
    if (blocks * kThreads >= 4294967296.0) return -2;
    const dim3 grid((unsigned)blocks, 2);
    if (few && p.c.D == 128) hipLaunchKernelGGL(kv_read_few<128>, grid, dim3(kThreads), 0, stream, p);
    else if (few) hipLaunchKernelGGL(kv_read_few<64>, grid, dim3(kThreads), 0, stream, p);
    else if (p.c.D == 128) hipLaunchKernelGGL(kv_read<128>, grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL(kv_read<64>, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
