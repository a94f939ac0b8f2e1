// Writing the quantised cache and reading it back, for gfx950.
//
// A workgroup owns the keys or the values of one page and kv head, so the page's exponent, its earlier tokens' codes and
// its new ones are one workgroup's business.  What bounds both: reading and writing every value once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "kv_launch.h"

namespace {

using namespace gfx950;

constexpr int kThreads = 256;
constexpr int kLeastExp = -100;

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }    // -126 <= e <= 127
__device__ __forceinline__ unsigned char to_e4m3(float x) {
    return (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
}
__device__ __forceinline__ float from_e4m3(unsigned char c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
__device__ __forceinline__ float bf16_bits(unsigned short b) { return __uint_as_float((unsigned)b << 16); }

// The least e >= kLeastExp with amax <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_for(float amax) {
    const unsigned bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kLeastExp ? kLeastExp : e;
}

template <int D>
__global__ __launch_bounds__(kThreads) void kv_write(KvWriteParams p) {
    constexpr int CPR = D / 8;
    __shared__ float s_max[kThreads / 64];
    const int tid = threadIdx.x, page = p.c.page;
    const bool is_v = blockIdx.y != 0;
    unsigned id = blockIdx.x;
    const int h = id % (unsigned)p.c.Hkv; id /= (unsigned)p.c.Hkv;
    const int f = id % (unsigned)p.F, b = id / (unsigned)p.F;

    const long long start = p.start[b];
    const int n = p.count ? min(max(p.count[b], 0), p.S) : p.S;
    const long long pg = (start >> p.c.page_log2) + f;                 // (arithmetic shift: rounds down)
    if (pg < 0 || pg >= p.c.W) return;
    const long long base = pg << p.c.page_log2;                        // the page's first position
    const long long lo = start > base ? start : base, hi = start + n < base + page ? start + n : base + page;
    if (lo >= hi) return;
    const int at = p.c.table[b * p.c.pitch + pg];
    if (at < 0 || at >= p.c.P) return;

    const int held = (int)(lo - base), fresh = (int)(hi - lo);         // earlier tokens of the page, new ones
    const __bf16* src = is_v ? p.v + b * p.v_sb + h * p.v_sh + (lo - start) * p.v_ss : p.k + b * p.k_sb + h * p.k_sh + (lo - start) * p.k_ss;
    const long long row = is_v ? p.v_ss : p.k_ss;
    const size_t unit = (size_t)at * p.c.Hkv + h;
    unsigned char* const codes = (is_v ? p.c.v : p.c.k) + unit * page * D;
    unsigned char* const exps = (is_v ? p.c.ve : p.c.ke) + unit;

    float amax = 0.f;
    for (int i = tid; i < fresh * CPR; i += kThreads) {
        const s16x8 x = *(const s16x8*)(src + (i / CPR) * row + (i % CPR) * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = fabsf(bf16_bits((unsigned short)x[j]));
            if (a < INFINITY) amax = fmaxf(amax, a);
        }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) amax = fmaxf(amax, __shfl_xor(amax, x));
    if ((tid & 63) == 0) s_max[tid >> 6] = amax;
    const int e_old = (int)*exps - 127;
    __syncthreads();
    amax = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    int e = exponent_for(amax);
    if (held > 0 && e < e_old) e = e_old;

    auto code_at = [&](int token, int d) { return codes + (is_v ? (size_t)d * page + token : (size_t)token * D + d); };
    if (held > 0 && e > e_old) {
        const float f2 = two_to(max(e_old - e, -126));
        for (int i = tid; i < held * D; i += kThreads) {
            unsigned char* const c = code_at(i / D, i % D);
            if ((*c & 0x7f) != 0x7f) *c = to_e4m3(from_e4m3(*c) * f2);
        }
    }
    const float f1 = two_to(-e);
    for (int i = tid; i < fresh * CPR; i += kThreads) {
        const s16x8 x = *(const s16x8*)(src + (i / CPR) * row + (i % CPR) * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = bf16_bits((unsigned short)x[j]);
            *code_at(held + i / CPR, (i % CPR) * 8 + j) = fabsf(a) < INFINITY ? to_e4m3(a * f1) : (unsigned char)0x7f;
        }
    }
    if (tid == 0) *exps = (unsigned char)(e + 127);
}

template <int D>
__global__ __launch_bounds__(kThreads) void kv_read(KvReadParams p) {
    constexpr int CPR = D / 8;
    const int page = p.c.page;
    const bool is_v = blockIdx.y != 0;
    const size_t idx = (size_t)blockIdx.x * kThreads + threadIdx.x;
    const int ch = idx % CPR;
    size_t r = idx / CPR;
    if (r >= (size_t)p.B * p.c.Hkv * p.S) return;
    const int s = r % (unsigned)p.S; r /= (unsigned)p.S;
    const int h = r % (unsigned)p.c.Hkv, b = r / (unsigned)p.c.Hkv;
    const long long pos = (long long)p.first + s;
    u32x4 w = {0, 0, 0, 0};
    if (pos < p.lens[b] && (pos >> p.c.page_log2) < p.c.W) {
        const int at = p.c.table[b * p.c.pitch + (pos >> p.c.page_log2)];
        if (at >= 0 && at < p.c.P) {
            const size_t unit = (size_t)at * p.c.Hkv + h;
            const unsigned char* const codes = (is_v ? p.c.v : p.c.k) + unit * page * D;
            const int token = (int)(pos & (page - 1));
            const int e = (int)(is_v ? p.c.ve : p.c.ke)[unit] - 127;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int d = ch * 8 + j;
                x[j] = ldexpf(from_e4m3(codes[is_v ? (size_t)d * page + token : (size_t)token * D + d]), e);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
        }
    }
    __bf16* const out = is_v ? p.v + b * p.v_sb + h * p.v_sh + s * p.v_ss : p.k + b * p.k_sb + h * p.k_sh + s * p.k_ss;
    *(u32x4*)(out + ch * 8) = w;
}

}  // namespace

int kv_write_launch(const KvWriteParams& p, hipStream_t stream) {
    const double blocks = (double)p.B * p.F * p.c.Hkv;
    if (blocks * kThreads >= 4294967296.0) return -2;
    const dim3 grid((unsigned)blocks, 2);
    if (p.c.D == 128) hipLaunchKernelGGL(kv_write<128>, grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL(kv_write<64>, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int kv_read_launch(const KvReadParams& p, hipStream_t stream) {
    const double threads = (double)p.B * p.c.Hkv * p.S * (p.c.D / 8);
    if (threads >= 4294967296.0 - kThreads) return -2;
    const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads), 2);
    if (p.c.D == 128) hipLaunchKernelGGL(kv_read<128>, grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL(kv_read<64>, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
