"""Shared helpers of the tests of the quantised cache: plain implementations in 64 bits, and caches to run on (not collected by pytest)."""
from __future__ import annotations

import math

import numpy as np

LEAST_EXP = -100


def e4m3_table():
    """What each of the 256 codes stands for (OCP e4m3)."""
    out = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        size = math.nan if (e, m) == (15, 7) else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out[code] = -size if code & 128 else size
    return out


E4M3 = e4m3_table()


def bf16(x):
    """x rounded to bf16 (ties to even), as 64-bit values; NaN stays NaN."""
    with np.errstate(over="ignore"):
        b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)) << np.uint64(16)
    return np.where(np.isnan(x), np.nan, r.astype(np.uint32).view(np.float32).astype(np.float64))


def quantise(x, e):
    """The codes of x / 2^e: nearest, ties to the even code; NaN and infinities are 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    y = np.where(np.isfinite(x), np.abs(x), 0.0) * 2.0 ** -float(e)
    sizes = E4M3[:127]                                               # 0 ... 448, ascending
    up = np.clip(np.searchsorted(sizes, y), 0, 126)
    down = np.maximum(up - 1, 0)
    closer_down = (y - sizes[down] < sizes[up] - y) | ((y - sizes[down] == sizes[up] - y) & (down % 2 == 0))
    code = np.where(closer_down, down, up).astype(np.uint8)
    code |= np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def least_exponent(amax):
    """The least e >= LEAST_EXP with amax <= 448 * 2^e."""
    e = LEAST_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def write_reference(cache, k, v, table, start, count):
    """kv_fp8_write on numpy arrays: cache = (k, v, k_exp, v_exp), changed in place; k, v [B, Hkv, S, D]."""
    P, H, page, D = cache[0].shape
    B, _, S, _ = k.shape
    for b in range(B):
        n = S if count is None else min(max(int(count[b]), 0), S)
        first = int(start[b])
        for slot in range(max(first, 0) // page, table.shape[1]):
            lo, hi = max(first, slot * page), min(first + n, (slot + 1) * page)
            at = int(table[b, slot])
            if lo >= hi or not 0 <= at < P:
                continue
            for h in range(H):
                for codes, exps, x in ((cache[0][at, h], cache[2], k), (cache[1][at, h].T, cache[3], v)):
                    new = x[b, h, lo - first:hi - first].astype(np.float64)
                    fin = np.abs(new[np.isfinite(new)])
                    e = least_exponent(fin.max() if fin.size else 0.0)
                    held = lo - slot * page
                    if held:
                        old = int(exps[at, h]) - 127
                        if old >= e:
                            e = old
                        else:
                            was = codes[:held].copy()
                            again = quantise(E4M3[was] * 2.0 ** float(old - e), 0)
                            codes[:held] = np.where((was & 0x7F) == 0x7F, was, again)
                    codes[held:held + hi - lo] = quantise(new, e)
                    exps[at, h] = e + 127


def gather_reference(cache, table, b, h, n):
    """Keys and values [n, D] of a sequence and head in 64 bits, and which positions are there."""
    P, _, page, D = cache[0].shape
    k, v, there = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n, dtype=bool)
    for slot in range(min(-(-n // page), table.shape[1])):
        at, m = int(table[b, slot]), min(page, n - slot * page)
        if 0 <= at < P:
            s = slice(slot * page, slot * page + m)
            k[s] = E4M3[cache[0][at, h]][:m] * 2.0 ** (float(cache[2][at, h]) - 127)
            v[s] = E4M3[cache[1][at, h]].T[:m] * 2.0 ** (float(cache[3][at, h]) - 127)
            there[s] = True
    return k, v, there


def attn_reference(q, cache, table, lens, q_lens, causal, window, sinks, scale):
    """(O, LSE, tolerance of O, tolerance of LSE) of attn_kv_fp8 in 64 bits.

    The tolerance counts the kernel's roundings: the probabilities to bf16 (2^-8 of each, so 2^-8 of sum p |v|), O to bf16
    (2^-8 |o|), and the fp32 score: a sum of D products (D + 8 half steps of sum |q k|), its scaled exponent and the
    exponential (a few units of 2^-24 of the score's size, 2^-20 in all)."""
    B, Hq, Sq, D = q.shape
    H = cache[0].shape[1]
    o, tol_o = np.zeros((B, Hq, Sq, D)), np.zeros((B, Hq, Sq, D))
    lse, tol_l = np.full((B, Hq, Sq), -np.inf), np.zeros((B, Hq, Sq))
    for b in range(B):
        n = max(0, min(int(lens[b]), table.shape[1] * cache[0].shape[2]))
        rows = Sq if q_lens is None else min(max(int(q_lens[b]), 0), Sq)
        for hk in range(H):
            k, v, there = gather_reference(cache, table, b, hk, n)
            j = np.arange(n)
            for h in range(hk * (Hq // H), (hk + 1) * (Hq // H)):
                for i in range(rows):
                    pos = n - rows + i
                    see = there.copy()
                    if causal:
                        see &= j <= pos
                    if window:
                        see &= (j > pos - window) | (j < sinks)
                    if not see.any():
                        continue
                    x = q[b, h, i].astype(np.float64)
                    s = scale * (k[see] @ x)
                    top = s.max()
                    p = np.exp(s - top)
                    total = p.sum()
                    w = p / total
                    size = scale * (np.abs(k[see]) @ np.abs(x)).max()
                    ds = (D + 8) * 2.0 ** -24 * size + 2.0 ** -22 * np.abs(s).max()
                    a = w @ np.abs(v[see])
                    o[b, h, i], lse[b, h, i] = w @ v[see], top + np.log(total)
                    tol_o[b, h, i] = 2.0 ** -8 * (a + np.abs(o[b, h, i])) + (2 * ds + 2.0 ** -20) * a + 1e-30
                    tol_l[b, h, i] = ds + 2.0 ** -20 + 2.0 ** -22 * abs(lse[b, h, i])
    return o, lse, tol_o, tol_l


def make_table(rng, lens, page, spare=2, width=None):
    """(table, pages): every sequence's pages, in no order."""
    need = [-(-max(int(n), 0) // page) for n in lens]
    width = max(max(need), 1) if width is None else width
    P = sum(need) + spare
    order = rng.permutation(P)
    table, at = np.full((len(lens), width), -1, dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, P


def make_cache(rng, P, H, page, D, spread=2):
    """A cache with normal values whose size differs from page to page; no NaN."""
    shape = (P, H)
    ke, ve = (rng.integers(127 - spread - 7, 127 + spread - 7, shape).astype(np.uint8) for _ in range(2))
    codes = lambda *s: quantise(np.clip(rng.standard_normal(s) * 100, -448, 448), 0)
    return [codes(P, H, page, D), codes(P, H, D, page), ke, ve]


def spoil_behind(cache, table, lens):
    """NaN codes at every position that no sequence holds, and in the pages of none."""
    P, H, page, D = cache[0].shape
    held = np.zeros((P, page), dtype=bool)
    for b in range(table.shape[0]):
        for slot in range(table.shape[1]):
            at = int(table[b, slot])
            if 0 <= at < P:
                held[at, :max(0, min(page, int(lens[b]) - slot * page))] = True
    cache[0][np.broadcast_to(~held[:, None, :, None], cache[0].shape)] = 0x7F
    cache[1][np.broadcast_to(~held[:, None, None, :], cache[1].shape)] = 0xFF


def to_cuda(cache, table):
    import torch
    from paper_2604_18616_amd import binding
    return binding.KvFp8Cache(*(torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in cache)), torch.from_numpy(table).cuda()


def whole(values):
    import torch
    return None if values is None else torch.tensor([int(v) for v in values], dtype=torch.int32, device="cuda")


def bf16_cuda(x):
    import torch
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def host(t):
    import torch
    return t.float().cpu().numpy().astype(np.float64) if t.dtype == torch.bfloat16 else t.cpu().numpy()
