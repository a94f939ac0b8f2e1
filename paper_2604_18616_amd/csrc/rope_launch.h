// Internal interface between the argument checks (rope_api.cpp) and the kernel (rope_kernel.hip).
#pragma once
#include <hip/hip_runtime.h>

struct RopeTensor {
    const __bf16* in;
    __bf16* out;
    long long in_sb, in_sh, in_ss, out_sb, out_sh, out_ss;   // element strides: batch, head, row
    int heads;
};
struct RopeParams {
    RopeTensor t[2];           // q, k (k.heads 0: none)
    const int* positions;
    long long pos_pitch;
    const double* inv_freq;
    int B, S, D, R;
    float mscale;
    float sign;                // -1: the inverse rotation
    int items;                 // threads per token (set by the launcher)
    int per;                   // heads per thread, of q's and k's one after the other (set by the launcher)
};

// Enqueue the kernel; 0, or -1 if the runtime refused the launch.
int rope_launch(RopeParams p, int interleaved, hipStream_t stream);
