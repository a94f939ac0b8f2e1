// Rotary position embedding for gfx950.
//
// A thread owns V pairs of columns of one token (or columns that are only copied) and walks heads, those of q and k as one
// range: the angle is the same for all of them, so its sine and cosine are made once, in registers, and no table is read.
// What bounds it: reading and writing every value once.  40 heads of 16384 tokens, all 128 columns turned (336 MB in and out),
// 65.6 us = 5.1 TB/s, where a copy of torch reaches 4.9; 32 heads of 8192 tokens, half the columns turned, 27 us = 5.0 TB/s;
// 40 heads of 64 tokens 3.1 us in a captured graph: latency.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gfx950_prims.h"
#include "rope_launch.h"

namespace {

using namespace gfx950;

constexpr int kThreads = 256;
// Heads per thread, and workgroups that a call should have at the least, so that loads of several of them are in flight on
// every CU: with 40 heads of 16384 tokens 8 / 20 / 4 / 1 heads take 69 / 79 / 78 / 90 us, with 48 heads of 4096 tokens
// 6 / 2 / 1 parts of the heads (1152 / 384 / 192 workgroups) 26 / 42 / 61 us.
constexpr int kHeads = 8, kLeastBlocks = 768;
// Results are not read again here.  Rows that one instruction stores whole (neighbours) go past the caches, 40 heads of 16384
// tokens 67.6 -> 65.9 us; halves are put together in L2: stored past it, 32 heads of 27720 tokens, 16 of 64 columns turned, take
// 113 us in place of 62 (and 145 where turned and copied columns are not stored side by side in one loop).
// Values are loaded past the caches where there are more than the memory-side cache keeps until they could be used again (72
// heads of 30000 tokens 199 -> 192 us, but 48 of 4096, which repeated calls find there, 19 -> 25).
constexpr double kStreamed = 128e6;

template <int N> struct Chunk;                          // N bf16 values as one access
template <> struct Chunk<8> { using type = u32x4; };
template <> struct Chunk<4> { using type = u32x2; };
template <> struct Chunk<2> { using type = unsigned; };
template <> struct Chunk<1> { using type = unsigned short; };

template <int N, bool ST>
__device__ __forceinline__ typename Chunk<N>::type fetch(const __bf16* p) {
    const auto* const from = (const typename Chunk<N>::type*)p;
    if constexpr (ST) return __builtin_nontemporal_load(from);
    else return *from;
}
template <int N>
__device__ __forceinline__ void values(typename Chunk<N>::type raw, float (&x)[N]) {
    typedef __attribute__((ext_vector_type(N))) unsigned short bits_t;
    const bits_t b = __builtin_bit_cast(bits_t, raw);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float((unsigned)b[i] << 16);
}
template <int N>
__device__ __forceinline__ typename Chunk<N>::type rounded(const float (&x)[N]) {
    typedef __attribute__((ext_vector_type(N))) float f_t;
    typedef __attribute__((ext_vector_type(N))) __bf16 b_t;
    f_t f;
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = x[i];
    return __builtin_bit_cast(typename Chunk<N>::type, __builtin_convertvector(f, b_t));
}
template <int N, bool PAST>
__device__ __forceinline__ void store(__bf16* p, typename Chunk<N>::type raw) {
    auto* const to = (typename Chunk<N>::type*)p;
    if constexpr (PAST) __builtin_nontemporal_store(raw, to);
    else *to = raw;
}

// x0 a + x1 b, in one order of roundings wherever it stands: a result does not depend on the other heads and tokens of a call.
__device__ __forceinline__ float turned(float x0, float a, float x1, float b) { return fmaf(x0, a, x1 * b); }

// Halves (IL false): pairs (f, f + R/2), two accesses of V values per head.  Neighbours (IL true): pairs (2f, 2f + 1), one
// access of 2 V values.
template <int V, bool IL, bool ST>
__global__ __launch_bounds__(kThreads) void rope_turn(RopeParams p) {
    const unsigned idx = blockIdx.x * kThreads + threadIdx.x, token = idx / (unsigned)p.items, item = idx % (unsigned)p.items;
    if (token >= (unsigned)p.B * (unsigned)p.S) return;
    const int b = token / (unsigned)p.S, s = token % (unsigned)p.S;
    const int first = (int)blockIdx.y * p.per, last = first + p.per;
    // each of this thread's heads of q, then of k, as the function's two rows
    auto heads = [&](auto&& turn) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const RopeTensor& t = p.t[x];
            const int before = x ? p.t[0].heads : 0, h0 = max(first - before, 0), h1 = min(last - before, t.heads);
            const __bf16* in = t.in + b * t.in_sb + h0 * t.in_sh + s * t.in_ss;
            __bf16* out = t.out + b * t.out_sb + h0 * t.out_sh + s * t.out_ss;
#pragma unroll 2
            for (int h = h0; h < h1; ++h, in += t.in_sh, out += t.out_sh) turn(in, out);
        }
    };

    // turned columns: pairs f ... f + V - 1; behind them copies.  Both in one stream, so that rows are read and written whole.
    constexpr int W = IL ? 2 * V : V;
    const int f = item * V;
    const bool turns = f < p.R / 2;
    const int col = turns ? (IL ? 2 * f : f) : p.R + (item - p.R / 2 / V) * W, other = p.R / 2 + f;
    float c[V] = {}, sn[V] = {};
    if (turns) {
        const double pos = (double)p.positions[b * p.pos_pitch + s];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const double angle = pos * (p.inv_freq[f + i] * 0.15915494309189533577);      // in turns
            const float part = (float)(angle - rint(angle));       // of a turn, in [-1/2, 1/2]
            sincospif(2.f * part, &sn[i], &c[i]);
            c[i] *= p.mscale;
            sn[i] *= p.mscale * p.sign;
        }
    }
    heads([&](const __bf16* in, __bf16* out) __attribute__((always_inline)) {
        typename Chunk<W>::type first = fetch<W, ST>(in + col);
        if constexpr (IL) {
            float x[W], y[W];
            values<W>(first, x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[2 * i] = turned(x[2 * i], c[i], -x[2 * i + 1], sn[i]);
                y[2 * i + 1] = turned(x[2 * i], sn[i], x[2 * i + 1], c[i]);
            }
            if (turns) first = rounded<W>(y);
        } else if (turns) {
            float x0[V], x1[V], y0[V], y1[V];
            values<V>(first, x0);
            values<V>(fetch<V, ST>(in + other), x1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y0[i] = turned(x0[i], c[i], -x1[i], sn[i]);
                y1[i] = turned(x0[i], sn[i], x1[i], c[i]);
            }
            first = rounded<V>(y0);
            store<V, IL>(out + other, rounded<V>(y1));
        }
        store<W, IL>(out + col, first);
    });
}

template <int V, bool IL>
void launch(RopeParams p, hipStream_t stream) {
    const bool in_place = p.t[0].in == p.t[0].out && (p.t[1].heads == 0 || p.t[1].in == p.t[1].out);
    p.items = p.R / 2 / V + (in_place ? 0 : (p.D - p.R) / (IL ? 2 * V : V));
    const long long tokens = (long long)p.B * p.S;
    const int all = p.t[0].heads + p.t[1].heads;
    const unsigned blocks = (unsigned)((tokens * p.items + kThreads - 1) / kThreads);
    const long long parts = std::max((all + kHeads - 1) / kHeads, (int)((kLeastBlocks + blocks - 1) / blocks));
    p.per = (int)((all + parts - 1) / parts);
    const dim3 grid(blocks, (all + p.per - 1) / p.per);
    const bool streamed = (double)tokens * all * p.D * 2 * sizeof(__bf16) > kStreamed;
    if (streamed) hipLaunchKernelGGL((rope_turn<V, IL, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((rope_turn<V, IL, false>), grid, dim3(kThreads), 0, stream, p);
}

}  // namespace

// The widest access that the pairs allow.
int rope_launch(RopeParams p, int interleaved, hipStream_t stream) {
    const int pairs = p.R / 2;
    if (interleaved) {
        if (pairs % 4 == 0) launch<4, true>(p, stream);
        else if (pairs % 2 == 0) launch<2, true>(p, stream);
        else launch<1, true>(p, stream);
    } else {
        if (pairs % 8 == 0) launch<8, false>(p, stream);
        else if (pairs % 4 == 0) launch<4, false>(p, stream);
        else if (pairs % 2 == 0) launch<2, false>(p, stream);
        else launch<1, false>(p, stream);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
