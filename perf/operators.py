"""Performance cases of the quantised cache and the operators around it, and the same operators in plain torch.

Four operators, in the order a layer uses them: rotary positions (``rope_bf16``), writing keys and values into a paged cache
of 8-bit codes (``kv_fp8_write``), attention over that cache (``attn_kv_fp8``, with a causal mask, a sliding window and a few
first tokens that stay visible) and reading the cache back (``kv_fp8_read``).

The cache: pages of ``page`` tokens, e4m3 codes k [P, Hkv, page, D] and v [P, Hkv, D, page], and for each page and kv head one
byte e + 127 for the keys and one for the values; a code c stands for c * 2^e.  Position j of sequence b is token j % page of
page table[b][j / page].

With ``own`` the library's entry points are called; without it elementary torch operations compute the same in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

LEAST_EXP = -100                       # the smallest exponent of a page: its codes are normal bf16 numbers once decoded
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _attn(B, Hq, Hkv, D, Sq, L, page, ragged=False, ragged_q=False, causal=True, window=0, sinks=0):
    return dict(op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, Sq=Sq, L=L, page=page, ragged=ragged, ragged_q=ragged_q,
                causal=causal, window=window, sinks=sinks)


def _write(B, H, D, S, L, page, ragged=False):
    """S new tokens of each sequence behind up to L - S held ones; ragged: fewer new tokens for some."""
    return dict(op="write", B=B, H=H, D=D, S=S, L=L, page=page, ragged=ragged)


def _read(B, H, D, L, page, ragged=False):
    return dict(op="read", B=B, H=H, D=D, L=L, page=page, ragged=ragged)


def _rope(B, S, Hq, Hk, D, R, interleaved, inverse=False, factor=1.0, layout="bshd"):
    return dict(op="rope", B=B, S=S, Hq=Hq, Hk=Hk, D=D, R=R, interleaved=interleaved, inverse=inverse, factor=factor, layout=layout)


def listed():
    return [
        # one sequence decodes, a short cache in small pages: latency counts
        dict(_attn(1, 32, 8, 128, 1, 2000, 16), name="attn_one_token"),
        # one decoding step of a batch whose caches have all lengths up to 8191
        dict(_attn(32, 32, 8, 128, 1, 8191, 64, ragged=True), name="attn_batch"),
        # one GPU's share of the heads against one very long cache
        dict(_attn(1, 8, 1, 128, 1, 131071, 128), name="attn_long"),
        # up to four speculated tokens of a batch, a window of 4096 tokens and four first ones that stay visible
        dict(_attn(16, 16, 16, 64, 4, 20000, 32, ragged=True, ragged_q=True, window=4096, sinks=4), name="attn_window"),
        # chunked prefill: 1000 new tokens of two prompts against long caches
        dict(_attn(2, 32, 8, 128, 1000, 16301, 64, ragged=True), name="attn_chunk"),
        # a decoding step's new token of each of 64 sequences
        dict(_write(64, 8, 128, 1, 8192, 16), name="write_step"),
        # prompts of up to 4096 tokens, some behind a cached beginning that ends inside a page
        dict(_write(4, 8, 128, 4096, 6000, 64, ragged=True), name="write_prompt"),
        # a few short caches of many narrow heads, read back
        dict(_read(2, 16, 64, 333, 16), name="read_short"),
        # the caches of a batch, read back as bf16
        dict(_read(8, 8, 128, 4001, 64, ragged=True), name="read_batch"),
        # a decoding step of 64 sequences, q and k together
        dict(_rope(64, 1, 32, 8, 128, 128, False), name="rope_step"),
        # a long prompt, neighbouring columns in pairs, frequencies stretched for a context eight times as long
        dict(_rope(1, 16384, 32, 8, 128, 128, True, factor=8.0), name="rope_prompt"),
        # the gradient of a training batch: the inverse rotation of half of each head
        dict(_rope(4, 2048, 16, 16, 128, 64, False, inverse=True, layout="bhsd"), name="rope_gradient"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    largest = {}
    for case in listed():
        for key, value in work(case).items():
            largest[key] = max(largest.get(key, 0), value)
    while True:
        case = _draw_any(rng)
        if all(value <= largest[key] for key, value in work(case).items()):
            return case


def _draw_any(rng):
    kind = rng.choice(("decode", "decode", "few", "chunk", "window", "write_step", "write_prompt", "read", "rope", "rope"))
    hkv = rng.choice((1, 2, 4, 8, 16))
    group = rng.choice((1, 2, 3, 4, 5, 8, 16))
    D = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 128))
    if kind in ("decode", "few", "chunk", "window"):
        L = _log_int(rng, 1, 131072)
        B = _log_int(rng, 1, max(1, min(128, (1 << 18) // L)))
        Sq = {"decode": 1, "few": rng.randint(2, 16), "chunk": _log_int(rng, 17, 2048), "window": rng.choice((1, 1, 3, 300))}[kind]
        Sq = min(Sq, L)
        window = _log_int(rng, 1, 8192) if kind == "window" else 0
        return _attn(B, hkv * group, hkv, D, Sq, L, page, ragged=rng.random() < 0.6, ragged_q=Sq > 1 and rng.random() < 0.3,
                     causal=Sq == 1 or rng.random() < 0.85, window=window, sinks=rng.choice((0, 1, 4, 70)) if window else 0)
    if kind == "write_step":
        return _write(_log_int(rng, 1, 256), hkv, D, rng.choice((1, 1, 2, 5)), _log_int(rng, 16, 2048), page, rng.random() < 0.5)
    if kind == "write_prompt":
        S = _log_int(rng, 6, 16384)
        return _write(_log_int(rng, 1, max(1, 32768 // S)), hkv, D, S, S + rng.choice((0, 1, 100, 1000)), page, rng.random() < 0.5)
    if kind == "read":
        L = _log_int(rng, 1, 32768)
        return _read(_log_int(rng, 1, max(1, 65536 // L)), hkv, D, L, page, rng.random() < 0.5)
    S = rng.choice((1, _log_int(rng, 1, 16384)))
    R = rng.choice((D, D, D // 2, D // 4, 16, 24, 20))
    return _rope(_log_int(rng, 1, max(1, min(256, 32768 // S))), S, hkv * group, hkv, D, R, rng.random() < 0.5, rng.random() < 0.3,
                 rng.choice((1.0, 4.0, 8.0, 32.0)), rng.choice(("bshd", "bhsd")))


def _spread(n, most, ragged):
    """n lengths up to `most`: all the same, or spread evenly down to one, in no order."""
    if not ragged or n == 1:
        return [most] * n
    step = next(k for k in (5, 7, 11, 13) if math.gcd(k, n) == 1 or k == 13)
    return [1 + (most - 1) * (n - (i * step) % n) // n for i in range(n)]


def _lens(c):
    """Keys and query rows of each sequence."""
    lens = _spread(c["B"], c["L"], c["ragged"])
    rows = [min(r, n) for r, n in zip(_spread(c["B"], c["Sq"], c["ragged_q"]), lens)] if c["ragged_q"] or c["ragged"] else [c["Sq"]] * c["B"]
    return lens, rows


def _new(c):
    """Tokens held before the call and new ones of each sequence."""
    count = _spread(c["B"], c["S"], c["ragged"])
    return [(c["L"] - c["S"]) * (1 + (3 * b) % 7) // 7 for b in range(c["B"])], count


def _below(n):
    """0 + 1 + ... + n - 1 for n > 0, else 0."""
    return n * (n - 1) // 2 if n > 0 else 0


def _visible(c, n, rows):
    """(query, key) pairs of one sequence and head, and keys that any row sees."""
    first = n - rows                                                  # position of row 0; rows end at position n - 1
    pairs = _below(n + 1) - _below(first + 1) if c["causal"] else rows * n
    keys = n if rows else 0
    w, s = c["window"], c["sinks"]
    if w:
        # row at position p loses the keys [sinks, p - window]: p - window - sinks + 1 of them where that is positive
        pairs -= _below(n - w - s + 1) - _below(first - w - s + 1)
        keys -= max(0, first - w - s + 1) if rows else 0
    return pairs, keys


def work(c):
    if c["op"] == "attn":
        lens, rows = _lens(c)
        seen = [_visible(c, n, r) for n, r in zip(lens, rows)]
        keys = sum(k for _, k in seen)
        return dict(bytes=2 * c["Hkv"] * c["D"] * keys + sum(rows) * c["Hq"] * c["D"] * 2 + c["B"] * c["Hq"] * c["Sq"] * (c["D"] * 2 + 4),
                    flops=4 * c["D"] * c["Hq"] * sum(p for p, _ in seen))
    if c["op"] == "write":
        values = 2 * sum(_new(c)[1]) * c["H"] * c["D"]
        return dict(bytes=3 * values, flops=2 * values)
    if c["op"] == "read":
        values = 2 * sum(_spread(c["B"], c["L"], c["ragged"])) * c["H"] * c["D"]
        return dict(bytes=values + 4 * c["B"] * c["L"] * c["H"] * c["D"], flops=values)
    values = c["B"] * c["S"] * (c["Hq"] + c["Hk"]) * c["D"]
    return dict(bytes=4 * values, flops=3 * values)


# ---------------------------------------------------------------------------------------------------------------
# preparation
# ---------------------------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e of whole numbers -126 ... 127, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(amax):
    """The least e >= LEAST_EXP with amax <= 448 * 2^e."""
    m, ex = torch.frexp(amax)
    e = torch.where(m <= E4M3_MAX / 512, ex - 9, ex - 8)
    return torch.where(amax > 0, e.clamp(min=LEAST_EXP), LEAST_EXP)


def _random_pages(gen, shape, token_dim):
    """Codes and exponents of pages that hold tokens: normal values whose size differs from page to page, a few columns
    larger than the others, as keys and values of a model have them."""
    P, H = shape[:2]
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16).float()
    x *= torch.exp(0.4 * torch.randn((P, H, 1, 1), generator=gen, device="cuda"))
    x.select(5 - token_dim, 3).mul_(4.0)
    e = _exponent(x.abs().amax((2, 3)))
    x *= _two_to(-e)[:, :, None, None]
    return x.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _make_cache(gen, lens, width, H, D, page):
    """A cache with the pages of sequences of these lengths, in no order, a few spare ones among them, and their table."""
    need = [-(-n // page) for n in lens]
    P = sum(need) + 3
    order = torch.randperm(P, generator=torch.Generator().manual_seed(int(gen.initial_seed()) % (1 << 31)))
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, ke = _random_pages(gen, (P, H, page, D), 2)
    v, ve = _random_pages(gen, (P, H, D, page), 3)
    return (k, v, ke, ve), table.cuda()


def _whole(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(gen, B, H, S, D, layout="bhsd"):
    """A [B, H, S, D] tensor, contiguous or a view of a [B, S, H, D] buffer."""
    shape = (B, H, S, D) if layout == "bhsd" else (B, S, H, D)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    return x if layout == "bhsd" else x.transpose(1, 2)


def _frequencies(c):
    """Radians per position of each pair of columns; for a context `factor` times as long, those that turn less than once in
    the original 4096 positions are slowed down by it, those that turn more than 32 times are kept."""
    f = 10000.0 ** (-torch.arange(0, c["R"], 2, dtype=torch.float64) / c["R"])
    if c["factor"] != 1.0:
        keep = ((4096 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        f = f * (keep + (1 - keep) / c["factor"])
    return f.cuda()


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(op=c["op"], case=c)
    if c["op"] == "attn":
        lens, rows = _lens(c)
        s["cache"], s["table"] = _make_cache(gen, lens, -(-c["L"] // c["page"]), c["Hkv"], c["D"], c["page"])
        s["q"] = _normal(gen, c["B"], c["Hq"], c["Sq"], c["D"], "bshd")
        s["lens"] = _whole(lens)
        s["q_lens"] = _whole(rows) if min(rows) < c["Sq"] else None
    elif c["op"] == "write":
        start, count = _new(c)
        s["cache"], s["table"] = _make_cache(gen, [a + n for a, n in zip(start, count)], -(-c["L"] // c["page"]), c["H"], c["D"], c["page"])
        s["k"], s["v"] = (_normal(gen, c["B"], c["H"], c["S"], c["D"], "bshd") for _ in range(2))
        s["start"] = _whole(start)
        s["count"] = _whole(count) if c["ragged"] else None
    elif c["op"] == "read":
        lens = _spread(c["B"], c["L"], c["ragged"])
        s["cache"], s["table"] = _make_cache(gen, lens, -(-c["L"] // c["page"]), c["H"], c["D"], c["page"])
        s["lens"] = _whole(lens)
    else:
        s["q"], s["k"] = (_normal(gen, c["B"], H, c["S"], c["D"], c["layout"]) for H in (c["Hq"], c["Hk"]))
        first = torch.randint(0, int(131072 * c["factor"]), (c["B"], 1), generator=gen, device="cuda", dtype=torch.int32)
        s["positions"] = (first + torch.arange(c["S"], device="cuda", dtype=torch.int32)).contiguous()
        s["inv_freq"] = _frequencies(c)
        s["scale"] = 1.0 if c["factor"] == 1.0 else 0.1 * math.log(c["factor"]) + 1.0     # what long contexts use against flat softmaxes
    return s


# ---------------------------------------------------------------------------------------------------------------
# the operators: the library's calls, or plain torch
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    return {"attn": _run_attn, "write": _run_write, "read": _run_read, "rope": _run_rope}[s["op"]](s)


def _run_attn(s):
    c = s["case"]
    if own:
        from paper_2604_18616_amd import KvFp8Cache, attn_kv_fp8
        return attn_kv_fp8(s["q"], KvFp8Cache(*s["cache"]), s["table"], s["lens"], q_lens=s["q_lens"], causal=c["causal"],
                           window=c["window"], sinks=c["sinks"])
    return _plain_attn(s["q"], s["cache"], s["table"], s["lens"], s["q_lens"], c["causal"], c["window"], c["sinks"])


def _run_write(s):
    k, v, k_exp, v_exp = s["cache"]
    if own:
        from paper_2604_18616_amd import KvFp8Cache, kv_fp8_write
        kv_fp8_write(KvFp8Cache(*s["cache"]), s["k"], s["v"], s["table"], s["start"], count=s["count"])
    else:
        _plain_write(s["cache"], s["k"], s["v"], s["table"], s["start"], s["count"])
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), k_exp, v_exp


def _run_read(s):
    c = s["case"]
    if own:
        from paper_2604_18616_amd import KvFp8Cache, kv_fp8_read
        return kv_fp8_read(KvFp8Cache(*s["cache"]), s["table"], s["lens"], c["L"])
    k, v, held = _plain_gather(s["cache"], s["table"], s["lens"])
    return tuple(torch.where(held[:, None, :, None], x, 0.0)[:, :, :c["L"]].to(torch.bfloat16) for x in (k, v))


def _run_rope(s):
    c = s["case"]
    if own:
        from paper_2604_18616_amd import rope_bf16
        return rope_bf16(s["q"], s["positions"], s["inv_freq"], k=s["k"], interleaved=c["interleaved"], inverse=c["inverse"], scale=s["scale"])
    return tuple(_plain_rope(x, s["positions"], s["inv_freq"], c["interleaved"], c["inverse"], s["scale"]) for x in (s["q"], s["k"]))


def _decoded(codes, exps):
    return codes.view(torch.float8_e4m3fn).float() * _two_to(exps.to(torch.int32) - 127)[..., None, None]


def _plain_gather(cache, table, lens):
    """Keys and values [B, Hkv, W * page, D] in 32 bits, and which positions are held."""
    k, v, ke, ve = cache
    P, H, page, D = k.shape
    B, W = table.shape
    known = (table >= 0) & (table < P)
    at = torch.where(known, table, 0).long()
    keys = _decoded(k[at], ke[at]).permute(0, 2, 1, 3, 4).reshape(B, H, W * page, D)
    values = _decoded(v[at], ve[at]).permute(0, 2, 1, 4, 3).reshape(B, H, W * page, D)
    j = torch.arange(W * page, device=table.device)
    return keys, values, (j < lens[:, None]) & known.repeat_interleave(page, 1)


def _plain_attn(q, cache, table, lens, q_lens, causal, window, sinks):
    keys, values, held = _plain_gather(cache, table, lens)
    values = torch.where(held[:, None, :, None], values, 0.0)
    B, Hq, Sq, D = q.shape
    H, n = keys.shape[1:3]
    rows = torch.full_like(lens, Sq) if q_lens is None else q_lens
    i, j = torch.arange(Sq, device=q.device), torch.arange(n, device=q.device)
    pos = (lens - rows)[:, None, None] + i[:, None]
    sees = held[:, None, :] & (i[:, None] < rows[:, None, None])
    if causal:
        sees = sees & (j <= pos)
    if window:
        sees = sees & ((j > pos - window) | (j < sinks))
    sees = sees[:, None, None]                                                            # [B, 1, 1, Sq, n]
    s = (q.float().reshape(B, H, Hq // H * Sq, D) @ keys.transpose(2, 3).contiguous()).reshape(B, H, Hq // H, Sq, n) * D ** -0.5
    s = torch.where(sees, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.where(sees, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(B, H, -1, n) @ values).reshape(B, H, -1, Sq, D) / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    return o.reshape(B, Hq, Sq, D).to(torch.bfloat16), lse.reshape(B, Hq, Sq)


def _plain_write(cache, k, v, table, start, count):
    """Pages that get new tokens are put together from old codes and new values, and written back."""
    P, H, page, D = cache[0].shape
    B, S = k.shape[0], k.shape[2]
    F = -(-S // page) + 1                                                                 # pages that S tokens can lie in
    frame = start[:, None] // page + torch.arange(F, device=k.device)                     # [B, F]
    at = torch.gather(table.long(), 1, frame.clamp(max=table.shape[1] - 1).long())
    pos = frame[:, :, None] * page + torch.arange(page, device=k.device)                  # [B, F, page]
    t = pos - start[:, None, None]
    n = torch.full_like(start, S) if count is None else count
    fresh = (t >= 0) & (t < n[:, None, None]) & (frame < table.shape[1])[:, :, None] & ((at >= 0) & (at < P))[:, :, None]
    old = pos < start[:, None, None]
    touched = fresh.any(2)                                                                # [B, F]
    t = t.clamp(0, S - 1).long().reshape(B, 1, F * page, 1).expand(B, H, F * page, D)
    held = old.any(2)
    for codes, exps, x, transposed in ((cache[0], cache[2], k, False), (cache[1], cache[3], v, True)):
        new = torch.gather(x, 2, t).float().reshape(B, H, F, page, D).transpose(1, 2)     # [B, F, H, page, D]
        seen = fresh[:, :, None, :, None]
        finite = torch.isfinite(new)
        e = _exponent(torch.where(seen & finite, new.abs(), 0.0).amax((3, 4)))            # [B, F, H]
        page_at = at.clamp(0, P - 1)
        e_old = exps[page_at].to(torch.int32) - 127
        e = torch.where(held[:, :, None], torch.maximum(e, e_old), e)
        before = codes[page_at]
        before = before.transpose(3, 4).contiguous() if transposed else before            # [B, F, H, page, D]
        again = (before.view(torch.float8_e4m3fn).float() * _two_to((e_old - e).clamp(min=-126))[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        coded = (new * _two_to(-e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        coded = torch.where(finite, coded, torch.full_like(coded, 0x7F))
        grown = (old[:, :, None, :] & (e > e_old)[..., None])[..., None]
        result = torch.where(seen, coded, torch.where(grown, again, before))
        codes[at[touched]] = (result.transpose(3, 4) if transposed else result)[touched]
        exps[at[touched]] = (e[touched] + 127).to(torch.uint8)


def _plain_rope(x, positions, inv_freq, interleaved, inverse, scale):
    R = 2 * inv_freq.numel()
    angle = positions.double()[:, None, :, None] * inv_freq
    cos, sin = (angle.cos() * scale).float(), (angle.sin() * (-scale if inverse else scale)).float()
    y = x.float()
    if interleaved:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, y[..., R:]), -1).to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    return {"attn": _exact_attn, "write": _exact_write, "read": _exact_read, "rope": _exact_rope}[c["op"]](s, c)


_E4M3 = None


def _e4m3_values():
    """What each of the 256 codes stands for."""
    global _E4M3
    if _E4M3 is None:
        def value(code):
            e, m = (code >> 3) & 15, code & 7
            size = math.nan if (e, m) == (15, 7) else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
            return -size if code & 128 else size
        _E4M3 = torch.tensor([value(code) for code in range(256)], dtype=torch.float64, device="cuda")
    return _E4M3


def _power(e):
    """2^e of whole numbers held in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_sequence(s, b, h, n):
    """The first n keys and values of one sequence and kv head, in 64 bits."""
    k, v, ke, ve = s["cache"]
    page = k.shape[2]
    at = s["table"][b, :-(-n // page)].long()
    keys = _e4m3_values()[k[at, h].long()] * _power(ke[at, h].long() - 127)[:, None, None]
    values = _e4m3_values()[v[at, h].long()] * _power(ve[at, h].long() - 127)[:, None, None]
    return keys.reshape(-1, k.shape[3])[:n], values.transpose(1, 2).reshape(-1, k.shape[3])[:n]


def _exact_attn(s, c):
    B, Hq, Sq, D, g = c["B"], c["Hq"], c["Sq"], c["D"], c["Hq"] // c["Hkv"]
    o = torch.zeros((B, Hq, Sq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, rows) in enumerate(zip(*_lens(c))):
        pos = torch.arange(n - rows, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None, :]
        hidden = (j > pos) if c["causal"] else torch.zeros((rows, n), dtype=torch.bool, device="cuda")
        if c["window"]:
            hidden = hidden | ((j <= pos - c["window"]) & (j >= c["sinks"]))
        for h in range(c["Hkv"]):
            keys, values = _exact_sequence(s, b, h, n)
            scores = torch.matmul(s["q"][b, h * g:(h + 1) * g, :rows].double(), keys.T.contiguous()) / math.sqrt(D)
            scores.masked_fill_(hidden, -math.inf)
            total = torch.logsumexp(scores, -1)
            lse[b, h * g:(h + 1) * g, :rows] = total
            o[b, h * g:(h + 1) * g, :rows] = torch.matmul(torch.exp(scores - total[..., None]), values)
    return o, lse


def _round_e4m3(x):
    """Multiples of the step that e4m3 has at this size, the nearest one, even ones on ties."""
    step = _power((torch.frexp(x.abs())[1] - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_write(s, c):
    page, codes = c["page"], _e4m3_values()
    k, v, ke, ve = s["cache"]
    table = s["table"].tolist()
    answers = []
    for x, held, exps, dims in ((s["k"], k, ke, (0, 1, 2)), (s["v"], v, ve, (0, 2, 1))):
        out = codes[held.long()]
        for b, (first, n) in enumerate(zip(*_new(c))):
            for f in range(first // page, (first + n - 1) // page + 1):
                lo, hi = max(first, f * page), min(first + n, (f + 1) * page)
                new = x[b, :, lo - first:hi - first].double()
                amax = new.abs().amax((1, 2))
                e = torch.floor(torch.log2(amax.clamp(min=1e-60) / E4M3_MAX)).long() - 1      # one or two too few
                e = e + (E4M3_MAX * _power(e) < amax).long()
                e = (e + (E4M3_MAX * _power(e) < amax).long()).clamp(min=LEAST_EXP)
                if lo > f * page:
                    before = exps[table[b][f]].long() - 127
                    e = torch.maximum(e, before)
                    part = out[table[b][f]].permute(dims)[:, :lo - f * page]
                    part.copy_(_round_e4m3(part * _power(before - e)[:, None, None]))
                out[table[b][f]].permute(dims)[:, lo - f * page:hi - f * page] = _round_e4m3(new * _power(-e)[:, None, None])
        answers.append(out)
    return answers[0], answers[1], None, None


def _exact_read(s, c):
    k, v = (torch.zeros((c["B"], c["H"], c["L"], c["D"]), dtype=torch.float64, device="cuda") for _ in range(2))
    for b, n in enumerate(_spread(c["B"], c["L"], c["ragged"])):
        for h in range(c["H"]):
            k[b, h, :n], v[b, h, :n] = _exact_sequence(s, b, h, n)
    return k, v


def _exact_rope(s, c):
    half = c["R"] // 2
    turn = torch.polar(torch.full((), s["scale"], dtype=torch.float64, device="cuda"), s["positions"].double()[:, None, :, None] * s["inv_freq"])
    turn = turn.conj() if c["inverse"] else turn
    answers = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        first, second = (slice(0, c["R"], 2), slice(1, c["R"], 2)) if c["interleaved"] else (slice(0, half), slice(half, c["R"]))
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        answers.append(y)
    return tuple(answers)
