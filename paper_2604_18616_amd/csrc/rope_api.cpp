// C ABI of the rotary position embedding: argument validation.  Every check runs before the first HIP call, so the
// error paths work on a machine without a GPU.  See include/rope.h for the contract.
#include <math.h>
#include <stdint.h>

#include "../../include/attn.h"
#include "../../include/rope.h"
#include "rope_launch.h"

static int check_strides(const long long* s, int D) {
    for (int i = 0; i < 3; ++i) {
        if (s[i] < 0 || s[i] >= (1LL << 40)) return ATTN_ERR_BAD_SHAPE;
        if (s[i] & 7) return ATTN_ERR_MISALIGNED;
    }
    return s[2] < D ? ATTN_ERR_BAD_SHAPE : ATTN_OK;
}

extern "C" int rope_bf16(const void* q, void* q_out, const void* k, void* k_out,
                         int B, int Hq, int Hk, int S, int D, int R,
                         const long long* q_strides, const long long* q_out_strides,
                         const long long* k_strides, const long long* k_out_strides,
                         const int* positions, long long positions_pitch, const double* inv_freq,
                         int interleaved, int inverse, float mscale, void* stream) {
    if (!q || !q_out || !q_strides || !q_out_strides || !positions || !inv_freq) return ATTN_ERR_NULL_PTR;
    if ((k != nullptr) != (Hk > 0) || (k_out != nullptr) != (Hk > 0)) return ATTN_ERR_NULL_PTR;
    if (Hk > 0 && (!k_strides || !k_out_strides)) return ATTN_ERR_NULL_PTR;
    if (B <= 0 || Hq <= 0 || Hk < 0 || S <= 0 || D <= 0) return ATTN_ERR_BAD_SHAPE;
    if ((long long)Hq + Hk > 65535 || positions_pitch < 0 || positions_pitch >= (1LL << 40)) return ATTN_ERR_BAD_SHAPE;
    if (D % 8 || D > 1024 || R < 2 || R % 2 || R > D) return ATTN_ERR_UNSUPPORTED;
    if ((double)B * S * D >= 2147483648.0) return ATTN_ERR_BAD_SHAPE;                  // threads are counted in 32 bits
    if (((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k | (uintptr_t)k_out) & 15u) return ATTN_ERR_MISALIGNED;
    if (((uintptr_t)positions & 3u) || ((uintptr_t)inv_freq & 7u)) return ATTN_ERR_MISALIGNED;
    if (int rc = check_strides(q_strides, D)) return rc;
    if (int rc = check_strides(q_out_strides, D)) return rc;
    if (Hk > 0) {
        if (int rc = check_strides(k_strides, D)) return rc;
        if (int rc = check_strides(k_out_strides, D)) return rc;
    }
    if (!isfinite(mscale)) return ATTN_ERR_BAD_SCALE;

    RopeParams p;
    auto tensor = [](const void* in, void* out, const long long* a, const long long* b, int heads) {
        return RopeTensor{(const __bf16*)in, (__bf16*)out, a[0], a[1], a[2], b[0], b[1], b[2], heads};
    };
    p.t[0] = tensor(q, q_out, q_strides, q_out_strides, Hq);
    p.t[1] = Hk > 0 ? tensor(k, k_out, k_strides, k_out_strides, Hk) : RopeTensor{};
    p.positions = positions; p.pos_pitch = positions_pitch; p.inv_freq = inv_freq;
    p.B = B; p.S = S; p.D = D; p.R = R;
    p.mscale = mscale; p.sign = inverse ? -1.f : 1.f;
    p.items = 0; p.per = 1;
    return rope_launch(p, interleaved != 0, (hipStream_t)stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

extern "C" int rope_frequencies(int R, double base, double factor, int original_len, double slow, double fast, double* inv_freq) {
    if (!inv_freq) return ATTN_ERR_NULL_PTR;
    if (R < 2 || R % 2 || original_len < 0) return ATTN_ERR_BAD_SHAPE;
    if (!(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor)) return ATTN_ERR_BAD_SCALE;
    if (original_len > 0 && (!(slow >= 0.0) || !(fast > slow) || !isfinite(fast))) return ATTN_ERR_BAD_SCALE;
    for (int f = 0; f < R / 2; ++f) {
        const double w = pow(base, -2.0 * f / R);
        double keep = 0.0;
        if (original_len > 0) {
            keep = (original_len * w / 6.283185307179586477 - slow) / (fast - slow);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        }
        inv_freq[f] = w * (keep + (1.0 - keep) / factor);
    }
    return ATTN_OK;
}
