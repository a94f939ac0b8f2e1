// C ABI of the quantised cache: argument validation and dispatch.  Every check below runs before the first HIP call, so the
// error paths work on a machine without a GPU.  See include/kv_cache.h for the contract.
#include <math.h>
#include <stdint.h>

#include "../../include/attn.h"
#include "../../include/kv_cache.h"
#include "kv_launch.h"

static int check_strides(const long long* s, int D) {
    if (s[2] < D || s[0] < 0 || s[1] < 0) return ATTN_ERR_BAD_SHAPE;           // rows may not overlap
    if ((s[0] | s[1] | s[2]) & 7) return ATTN_ERR_MISALIGNED;                  // keep every row 16-byte aligned
    return s[2] >= (1LL << 28) ? ATTN_ERR_BAD_SHAPE : ATTN_OK;
}

static int check_sizes(int Hkv, int D, int page) {
    if (Hkv <= 0 || D <= 0 || page <= 0) return ATTN_ERR_BAD_SHAPE;
    if (D != 64 && D != 128) return ATTN_ERR_UNSUPPORTED;
    return page == 16 || page == 32 || page == 64 || page == 128 ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

// The cache and its table, checked, as the kernels take them.
static int pages_of(const KvFp8Cache* c, const int* table, long long pitch, int width, KvPages* out) {
    if (!c || !c->k || !c->v || !c->k_exp || !c->v_exp || !table) return ATTN_ERR_NULL_PTR;
    if (c->pages <= 0 || width <= 0 || pitch < 0 || pitch >= (1LL << 40)) return ATTN_ERR_BAD_SHAPE;
    if (int rc = check_sizes(c->Hkv, c->D, c->page)) return rc;
    if ((long long)c->pages * c->Hkv >= (1LL << 31) || (long long)width * c->page >= (1LL << 30)) return ATTN_ERR_BAD_SHAPE;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15u || (uintptr_t)table & 3u) return ATTN_ERR_MISALIGNED;
    out->k = (unsigned char*)c->k; out->v = (unsigned char*)c->v; out->ke = c->k_exp; out->ve = c->v_exp;
    out->P = c->pages; out->Hkv = c->Hkv; out->page = c->page; out->D = c->D;
    out->page_log2 = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
    out->table = table; out->pitch = pitch; out->W = width;
    return ATTN_OK;
}

static int answer(int rc) { return rc == 0 ? ATTN_OK : rc == -2 ? ATTN_ERR_BAD_SHAPE : ATTN_ERR_LAUNCH; }

extern "C" int kv_fp8_write(const KvFp8Cache* cache, const void* k, const void* v, const long long* ks, const long long* vs,
                            const int* table, long long table_pitch, int width, const int* start, const int* count,
                            int B, int S, void* stream) {
    if (!k || !v || !ks || !vs || !start) return ATTN_ERR_NULL_PTR;
    KvWriteParams p;
    if (int rc = pages_of(cache, table, table_pitch, width, &p.c)) return rc;
    if (B <= 0 || S <= 0 || S >= (1 << 30)) return ATTN_ERR_BAD_SHAPE;
    if (((uintptr_t)k | (uintptr_t)v) & 15u || ((uintptr_t)start | (uintptr_t)count) & 3u) return ATTN_ERR_MISALIGNED;
    if (int rc = check_strides(ks, p.c.D)) return rc;
    if (int rc = check_strides(vs, p.c.D)) return rc;
    p.k = (const __bf16*)k; p.v = (const __bf16*)v;
    p.k_sb = ks[0]; p.k_sh = ks[1]; p.k_ss = ks[2];
    p.v_sb = vs[0]; p.v_sh = vs[1]; p.v_ss = vs[2];
    p.start = start; p.count = count; p.B = B; p.S = S;
    p.F = (S + p.c.page - 2) / p.c.page + 1;               // the first token may be the last of its page
    return answer(kv_write_launch(p, (hipStream_t)stream));
}

extern "C" int kv_fp8_read(const KvFp8Cache* cache, const int* table, long long table_pitch, int width, const int* lens,
                           void* k, void* v, const long long* ks, const long long* vs, int B, int S, int first, void* stream) {
    if (!k || !v || !ks || !vs || !lens) return ATTN_ERR_NULL_PTR;
    KvReadParams p;
    if (int rc = pages_of(cache, table, table_pitch, width, &p.c)) return rc;
    if (B <= 0 || S <= 0 || S >= (1 << 30) || first < 0) return ATTN_ERR_BAD_SHAPE;
    if (((uintptr_t)k | (uintptr_t)v) & 15u || (uintptr_t)lens & 3u) return ATTN_ERR_MISALIGNED;
    if (int rc = check_strides(ks, p.c.D)) return rc;
    if (int rc = check_strides(vs, p.c.D)) return rc;
    p.k = (__bf16*)k; p.v = (__bf16*)v;
    p.k_sb = ks[0]; p.k_sh = ks[1]; p.k_ss = ks[2];
    p.v_sb = vs[0]; p.v_sh = vs[1]; p.v_ss = vs[2];
    p.lens = lens; p.B = B; p.S = S; p.first = first;
    return answer(kv_read_launch(p, (hipStream_t)stream));
}

// Keys in the tiles of 64 that the rows of a workgroup see at the most: a window's and the first tokens' tiles begin and end anywhere.
static int keys_seen(int Sq, int max_len, int window, int sinks) {
    if (!window) return max_len;
    const long long keys = (long long)window + (sinks < max_len ? sinks : max_len) + Sq + 192;
    return keys < max_len ? (int)keys : max_len;
}

static size_t part_bytes(int B, int Hq, int Sq, int D, int splits) {
    return splits <= 1 ? 0 : (size_t)B * Hq * Sq * splits * (D + 2) * sizeof(float);
}

static int check_rows(int B, int Hq, int Hkv, int Sq) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Hq % Hkv != 0) return ATTN_ERR_BAD_SHAPE;
    if ((long long)(Hq / Hkv) * Sq >= (1LL << 28) || (double)B * Hq * Sq >= 2147483648.0) return ATTN_ERR_BAD_SHAPE;
    return ATTN_OK;
}

extern "C" size_t attn_kv_fp8_workspace_bytes(int B, int Hq, int Hkv, int Sq, int max_len, int D, int window, int sinks) {
    if (check_rows(B, Hq, Hkv, Sq) || check_sizes(Hkv, D, 16) || max_len <= 0 || max_len >= (1 << 30) || window < 0 || sinks < 0) return 0;
    return part_bytes(B, Hq, Sq, D, attn_kv_plan(B, Hq, Hkv, Sq, keys_seen(Sq, max_len, window, sinks), D, 0, 0).splits);
}

extern "C" int attn_kv_fp8(const void* q, const KvFp8Cache* cache, const int* table, long long table_pitch, int width,
                           const int* lens, const int* q_lens, void* o, float* lse, int B, int Hq, int Sq,
                           const long long* qs, const long long* os,
                           int causal, int window, int sinks, float scale, int max_len,
                           void* workspace, size_t workspace_bytes, int splits, int wg_rows, void* stream) {
    if (!q || !o || !lens || !qs || !os) return ATTN_ERR_NULL_PTR;
    KvAttnParams p;
    if (int rc = pages_of(cache, table, table_pitch, width, &p.c)) return rc;
    if (int rc = check_rows(B, Hq, p.c.Hkv, Sq)) return rc;
    if (window < 0 || sinks < 0 || max_len < 0) return ATTN_ERR_BAD_SHAPE;
    if (splits < 0 || splits > kMaxKvSplits || (wg_rows != 0 && wg_rows != 16 && wg_rows != 128)) return ATTN_ERR_UNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)o | (uintptr_t)workspace) & 15u) return ATTN_ERR_MISALIGNED;
    if (((uintptr_t)lse | (uintptr_t)lens | (uintptr_t)q_lens) & 3u) return ATTN_ERR_MISALIGNED;
    if (int rc = check_strides(qs, p.c.D)) return rc;
    if (int rc = check_strides(os, p.c.D)) return rc;
    if (!(scale > 0.0f) || scale > 1e38f) return ATTN_ERR_BAD_SCALE;   // rejects NaN, <= 0, and what the factor of base 2 would make infinite

    p.q = (const __bf16*)q; p.o = (__bf16*)o; p.lse = lse;
    p.q_sb = qs[0]; p.q_sh = qs[1]; p.q_ss = qs[2];
    p.o_sb = os[0]; p.o_sh = os[1]; p.o_ss = os[2];
    p.lens = lens; p.q_lens = q_lens;
    p.B = B; p.Hq = Hq; p.Sq = Sq;
    p.max_len = width * p.c.page;
    if (max_len > 0 && max_len < p.max_len) p.max_len = max_len;
    p.causal = causal != 0; p.window = window; p.sinks = sinks;
    p.scale = scale;
    p.scale_log2 = (float)((double)scale * 1.4426950408889634074);
    const int keys = keys_seen(Sq, p.max_len, window, sinks);
    KvAttnPlan plan = attn_kv_plan(B, Hq, p.c.Hkv, Sq, keys, p.c.D, splits, wg_rows);
    if (!workspace || workspace_bytes < part_bytes(B, Hq, Sq, p.c.D, plan.splits))
        plan = attn_kv_plan(B, Hq, p.c.Hkv, Sq, keys, p.c.D, 1, wg_rows);
    p.part = (float*)workspace;
    p.ml = plan.splits > 1 ? p.part + (size_t)B * Hq * Sq * plan.splits * p.c.D : nullptr;
    return answer(attn_kv_launch(p, plan, (hipStream_t)stream));
}
