// Internal interface between the argument checks (kv_api.cpp) and the kernels of the quantised cache (kv_cache_kernel.hip,
// attn_kv_kernel.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

struct KvPages {
    unsigned char *k, *v, *ke, *ve;
    int P, Hkv, page, page_log2, D;
    const int* table;
    long long pitch;
    int W;
};

struct KvWriteParams {
    KvPages c;
    const __bf16 *k, *v;
    long long k_sb, k_sh, k_ss, v_sb, v_sh, v_ss;
    const int *start, *count;      // count may be null
    int B, S;
    int F;                         // pages that S tokens can lie in
};

struct KvReadParams {
    KvPages c;
    __bf16 *k, *v;
    long long k_sb, k_sh, k_ss, v_sb, v_sh, v_ss;
    const int* lens;
    int B, S, first;
};

struct KvAttnParams {
    KvPages c;
    const __bf16* q;
    __bf16* o;
    float* lse;                    // may be null
    long long q_sb, q_sh, q_ss, o_sb, o_sh, o_ss;
    const int *lens, *q_lens;      // q_lens may be null
    int B, Hq, Sq, max_len;
    int causal, window, sinks;
    float scale, scale_log2;
    int row_wgs, splits;           // workgroups along the packed query rows of a kv head, and along its keys
    int most_tiles;                // that the rows of a workgroup can see
    float *part, *ml;              // [B*Hq*Sq, splits, D] and [B*Hq*Sq, splits, 2], as in attn_launch.h
};

// Each returns 0, -1 if the runtime refused the launch, -2 if the grid would not fit.
int kv_write_launch(const KvWriteParams& p, hipStream_t stream);
int kv_read_launch(const KvReadParams& p, hipStream_t stream);

// How a call's rows and keys are cut; splits, wg_rows 0: by size.  Host arithmetic only.
constexpr int kMaxKvSplits = 256;
struct KvAttnPlan { int rows, waves, row_wgs, splits, keys; };       // rows: packed query rows per workgroup; keys: that they can see
KvAttnPlan attn_kv_plan(int B, int Hq, int Hkv, int Sq, int keys, int D, int splits, int wg_rows);
int attn_kv_launch(KvAttnParams p, const KvAttnPlan& plan, hipStream_t stream);
