// Rotary position embedding for gfx950.
//
// A thread owns V pairs of columns of one token (or V columns that are only copied) and walks the heads: the angle is the
// same for all of them, so its sine and cosine are made once, in registers, and no table is read.  What bounds it: reading
// and writing every value once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "rope_launch.h"

namespace {

using namespace gfx950;

constexpr int kThreads = 256;
constexpr double kFull = 1 << 19;

template <int N> struct Chunk;                          // N bf16 values as one access
template <> struct Chunk<8> { using type = u32x4; };
template <> struct Chunk<4> { using type = u32x2; };
template <> struct Chunk<2> { using type = unsigned; };
template <> struct Chunk<1> { using type = unsigned short; };

template <int N>
__device__ __forceinline__ void load(const __bf16* p, float (&x)[N]) {
    typedef __attribute__((ext_vector_type(N))) unsigned short bits_t;
    const bits_t b = __builtin_bit_cast(bits_t, *(const typename Chunk<N>::type*)p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float((unsigned)b[i] << 16);
}
template <int N>
__device__ __forceinline__ void store(__bf16* p, const float (&x)[N]) {
    typedef __attribute__((ext_vector_type(N))) float f_t;
    typedef __attribute__((ext_vector_type(N))) __bf16 b_t;
    f_t f;
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = x[i];
    *(typename Chunk<N>::type*)p = __builtin_bit_cast(typename Chunk<N>::type, __builtin_convertvector(f, b_t));
}

// Halves (IL false): pairs (f, f + R/2), two accesses of V values per head.  Neighbours (IL true): pairs (2f, 2f + 1), one
// access of 2 V values.
template <int V, bool IL>
__global__ __launch_bounds__(kThreads) void rope_turn(RopeParams p) {
    const unsigned idx = blockIdx.x * kThreads + threadIdx.x, token = idx / (unsigned)p.items, item = idx % (unsigned)p.items;
    if (token >= (unsigned)p.B * (unsigned)p.S) return;
    const int b = token / (unsigned)p.S, s = token % (unsigned)p.S;
    const bool is_q = blockIdx.y < (unsigned)p.chunks_q;
    const RopeTensor& t = p.t[is_q ? 0 : 1];
    const int h0 = (int)(blockIdx.y - (is_q ? 0 : p.chunks_q)) * p.per, h1 = min(h0 + p.per, t.heads);
    const __bf16* in = t.in + b * t.in_sb + h0 * t.in_sh + s * t.in_ss;
    __bf16* out = t.out + b * t.out_sb + h0 * t.out_sh + s * t.out_ss;

    const int f = item * V;
    if (f >= p.R / 2) {                                 // behind the turned columns: copies
        constexpr int W = IL ? 2 * V : V;
        const int col = p.R + (item - p.R / 2 / V) * W;
        for (int h = h0; h < h1; ++h, in += t.in_sh, out += t.out_sh)
            *(typename Chunk<W>::type*)(out + col) = *(const typename Chunk<W>::type*)(in + col);
        return;
    }
    float c[V], sn[V];
    const double pos = (double)p.positions[b * p.pos_pitch + s];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const double turns = pos * (p.inv_freq[f + i] * 0.15915494309189533577);
        const float part = (float)(turns - rint(turns));       // of a turn, in [-1/2, 1/2]
        sincospif(2.f * part, &sn[i], &c[i]);
        c[i] *= p.mscale;
        sn[i] *= p.mscale * p.sign;
    }
#pragma unroll 4
    for (int h = h0; h < h1; ++h, in += t.in_sh, out += t.out_sh) {
        if constexpr (IL) {
            float x[2 * V], y[2 * V];
            load<2 * V>(in + 2 * f, x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * sn[i];
                y[2 * i + 1] = x[2 * i] * sn[i] + x[2 * i + 1] * c[i];
            }
            store<2 * V>(out + 2 * f, y);
        } else {
            float x0[V], x1[V], y0[V], y1[V];
            load<V>(in + f, x0);
            load<V>(in + p.R / 2 + f, x1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y0[i] = x0[i] * c[i] - x1[i] * sn[i];
                y1[i] = x0[i] * sn[i] + x1[i] * c[i];
            }
            store<V>(out + f, y0);
            store<V>(out + p.R / 2 + f, y1);
        }
    }
}

template <int V, bool IL>
void launch(RopeParams p, hipStream_t stream) {
    const bool in_place = p.t[0].in == p.t[0].out && (p.t[1].heads == 0 || p.t[1].in == p.t[1].out);
    p.items = p.R / 2 / V + (in_place ? 0 : (p.D - p.R) / (IL ? 2 * V : V));
    const long long tokens = (long long)p.B * p.S;
    // heads per thread: as many as leave the chip kFull threads
    const double threads = (double)tokens * p.items * (p.t[0].heads + p.t[1].heads);
    const int most = p.t[0].heads > p.t[1].heads ? p.t[0].heads : p.t[1].heads;
    p.per = threads < 2 * kFull ? 1 : threads / kFull < most ? (int)(threads / kFull) : most;
    p.chunks_q = (p.t[0].heads + p.per - 1) / p.per;
    const unsigned rows = p.chunks_q + (p.t[1].heads + p.per - 1) / p.per;
    const unsigned blocks = (unsigned)((tokens * p.items + kThreads - 1) / kThreads);
    hipLaunchKernelGGL((rope_turn<V, IL>), dim3(blocks, rows), dim3(kThreads), 0, stream, p);
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
