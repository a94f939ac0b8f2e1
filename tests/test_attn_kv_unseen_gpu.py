"""Attention over the quantised cache: what no row sees changes nothing, whatever its codes and exponents stand for."""
import ctypes

import numpy as np
import pytest

from _kv_util import attn_reference, bf16, bf16_cuda, host, make_cache, make_table, to_cuda, whole

pytestmark = pytest.mark.gpu


def call(q, cache, table, lens, q_lens=None, causal=True, window=0, sinks=0, splits=1, wg_rows=0):
    """The C entry point with memory for `splits` parts (0: the library's choice): O and LSE."""
    import torch
    from paper_2604_18616_amd import binding
    B, Hq, Sq, D = q.shape
    dev, tab = to_cuda(cache, table)
    struct, qd = binding._cache_struct(dev)[0], bf16_cuda(q)
    o, lse = torch.full_like(qd, float("nan")), torch.full((B, Hq, Sq), float("nan"), dtype=torch.float32, device="cuda")
    need = 4 * B * Hq * Sq * (splits or 256) * (D + 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    st, dl, dq = (ctypes.c_longlong * 3)(*qd.stride()[:3]), whole(lens), whole(q_lens)
    rc = binding.load_library().attn_kv_fp8(qd.data_ptr(), ctypes.byref(struct), tab.data_ptr(), tab.stride(0), tab.shape[1], dl.data_ptr(),
                                            None if dq is None else dq.data_ptr(), o.data_ptr(), lse.data_ptr(), B, Hq, Sq, st, st, int(causal), window, sinks,
                                            D ** -0.5, 0, ws.data_ptr(), need, splits, wg_rows, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return host(o), host(lse).astype(np.float64)


def check(got, want, what):
    (o, lse), (wo, wl, to, tl) = got, want
    gone = np.isneginf(wl)
    assert np.array_equal(np.isneginf(lse), gone), what
    assert np.all(np.abs(lse[~gone] - wl[~gone]) <= tl[~gone]), what
    assert np.all(np.abs(o - wo) <= to), (what, np.argwhere(~(np.abs(o - wo) <= to))[:4].tolist())


def unheld(cache, table, lens, code, exponent):
    """This code wherever no sequence holds a token, this exponent byte on the pages of none."""
    P, H, page, D = cache[0].shape
    held = np.zeros((P, page), dtype=bool)
    for b in range(table.shape[0]):
        for slot in range(table.shape[1]):
            if 0 <= table[b, slot] < P:
                held[table[b, slot], :max(0, min(page, int(lens[b]) - slot * page))] = True
    assert not held[0].any()
    cache[0][np.broadcast_to(~held[:, None, :, None], cache[0].shape)] = code
    cache[1][np.broadcast_to(~held[:, None, None, :], cache[1].shape)] = code
    for exps in cache[2:]:
        exps[~held.any(1)] = exponent


def with_null_page(rng, lens, page):
    """(table, pages) as make_table, but page 0 is no sequence's."""
    table, P = make_table(rng, lens, page)
    return np.where(table >= 0, table + 1, table).astype(np.int32), P + 1


@pytest.mark.parametrize("exponent,code", [(255, 0x7E), (255, 0x01), (255, 0x00), (255, 0xFF), (254, 0x7E), (248, 0x78), (247, 0xFE), (247, 0x7F), (0, 0x7E)])
@pytest.mark.parametrize("B,Hq,Hkv,D,Sq,lens,page", [
    (2, 4, 2, 128, 1, [70, 16], 16),
    (3, 8, 1, 64, 4, [1, 200, 385], 64),
    (1, 12, 2, 128, 20, [333], 32),
    (2, 4, 2, 64, 70, [97, 140], 128),
])
def test_pages_that_no_sequence_holds(B, Hq, Hkv, D, Sq, lens, page, exponent, code):
    """Lengths that leave groups of 16 keys of the last tile empty, and missing pages; page 0 belongs to nobody."""
    rng = np.random.default_rng(exponent + code + Sq)
    table, P = with_null_page(rng, lens, page)
    cache = make_cache(rng, P, Hkv, page, D)
    q = bf16(rng.standard_normal((B, Hq, Sq, D)))
    for missing in (False, True):
        if missing:
            table[:, 1::3] = -1
            table[0, 0] = P
        unheld(cache, table, lens, code, exponent)
        want = attn_reference(q, cache, table, lens, None, True, 0, 0, D ** -0.5)
        for wg_rows in (16, 128):
            for splits in (1, 3):
                print(missing, wg_rows, splits, flush=True)
                check(call(q, cache, table, lens, splits=splits, wg_rows=wg_rows), want, (missing, wg_rows, splits))


@pytest.mark.parametrize("exponent,code", [(255, 0x7E), (255, 0x00), (247, 0x78)])
@pytest.mark.parametrize("B,Hkv,D,most,least,page", [(200, 2, 64, 131, 0, 16), (200, 2, 128, 131, 0, 16), (32, 8, 128, 1500, 1, 32), (1, 1, 64, 2001, 0, 16)])
def test_pages_that_no_sequence_holds_in_batches(B, Hkv, D, most, least, page, exponent, code):
    """Shapes of decoding steps for which the library takes one, four and eight wavefronts, cut and not."""
    rng = np.random.default_rng(B + D + exponent)
    lens = [most] + [int(n) for n in rng.integers(least, 131, B - 1)]
    table, P = with_null_page(rng, lens, page)
    table[:, 2::5] = -1
    cache = make_cache(rng, P, Hkv, page, D)
    unheld(cache, table, lens, code, exponent)
    q = bf16(rng.standard_normal((B, 2 * Hkv, 1, D)))
    want = attn_reference(q, cache, table, lens, None, True, 0, 0, D ** -0.5)
    for splits in (0, 1, 8):
        print(splits, flush=True)
        check(call(q, cache, table, lens, splits=splits), want, splits)


def test_a_cache_as_it_is_allocated():
    """Memory that holds all ones before it is written, a null page, a prompt and a token: finite, and as the definition has it."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(7)
    D, page, lens = 64, 32, [37, 81]
    table, P = with_null_page(rng, [n + 1 for n in lens], page)
    cache = binding.kv_fp8_cache(P, 2, page, D)
    for t in cache:
        t.fill_(0xFF)
    tab, start = torch.from_numpy(table).cuda(), whole([0, 0])
    for S, counts in ((81, lens), (1, [1, 1])):
        k, v = (bf16_cuda(rng.standard_normal((2, 2, S, D))) for _ in range(2))
        q, count = bf16(rng.standard_normal((2, 4, S, D))), whole(counts)
        binding.kv_fp8_write(cache, k, v, tab, start, count=count)
        start = start + count
        torch.cuda.synchronize()
        want = attn_reference(q, [host(t) for t in cache], table, host(start), counts, True, 0, 0, D ** -0.5)
        for wg_rows in (0, 16, 128):
            o, lse = binding.attn_kv_fp8(bf16_cuda(q), cache, tab, start, q_lens=count, causal=True, wg_rows=wg_rows)
            torch.cuda.synchronize()
            check((host(o), host(lse).astype(np.float64)), want, (S, wg_rows))


# (position, column, code): 2^120 times 256 and more is infinite in bf16
def spoilt_value(cache, table, page, pos, d, code):
    """V of the page that holds a position at the largest exponent, its other codes small, this code at column d."""
    at = table[0, pos // page]
    if cache[3][at, 0] != 247:
        cache[3][at, 0] = 247
        cache[1][at, 0] &= 0x07                                 # 2^111 at the most: sums of them are finite
    cache[1][at, 0, d, pos % page] = code


@pytest.mark.parametrize("Sq,D,window", [(4, 128, 0), (4, 64, 30), (70, 128, 0), (200, 64, 40)])
@pytest.mark.parametrize("wg_rows,splits", [(16, 1), (16, 3), (128, 1), (128, 2)])
def test_infinite_values_reach_the_rows_that_see_them(Sq, D, window, wg_rows, splits):
    """Infinities among the last tokens, at a window's end, behind the last token and where every row sees them: the sign's
    infinity in their column for the rows that see one, NaN for those that see both, the other rows as if they were not there."""
    rng = np.random.default_rng(Sq + wg_rows + splits)
    n, page = Sq + 91, 16
    table, P = make_table(rng, [n], page)
    clean = make_cache(rng, P, 1, page, D)
    q = bf16(rng.standard_normal((1, 2, Sq, D)))
    row_pos = n - Sq + np.arange(Sq)
    for places in ([(n - 2, 5, 0x78)], [(n - Sq, D - 1, 0xFE)], [(n, 3, 0x7E)], [(70, 9, 0xF8)], [(3, 0, 0x7C)],
                   [(n - 1, 2, 0x7E), (n - 3, 2, 0xFE)], [(n - 2, 4, 0x7E), (n - 1, 4, 0x7F)]):
        spoilt, zeroed = [t.copy() for t in clean], [t.copy() for t in clean]
        up, down, nan = (np.zeros((Sq, D), dtype=bool) for _ in range(3))
        for pos, d, code in places:
            spoilt_value(spoilt, table, page, pos, d, code)
            spoilt_value(zeroed, table, page, pos, d, 0)
            sees = (pos <= row_pos) & ((pos > row_pos - window) if window else True) & (pos < n)
            (nan if code == 0x7F else down if code & 0x80 else up)[sees, d] = True
        nan |= up & down
        wo, wl, to, tl = attn_reference(q, zeroed, table, [n], None, True, window, 0, D ** -0.5)
        o, lse = call(q, spoilt, table, [n], window=window, splits=splits, wg_rows=wg_rows)
        for h in range(2):
            assert np.array_equal(np.isnan(o[0, h]), nan), places
            assert np.array_equal(np.isposinf(o[0, h]), up & ~nan) and np.array_equal(np.isneginf(o[0, h]), down & ~nan), places
            o[0, h][up | down | nan] = wo[0, h][up | down | nan]
        check((o, lse), (wo, wl, to, tl), places)


@pytest.mark.parametrize("Sq", [3, 60])
def test_the_largest_numbers_written_behind_the_mask(Sq):
    """A token of +-1.99 * 2^127, which the cache holds as infinities, as the last one: the rows before it do not see it."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(Sq)
    D, page, n = 128, 64, 130
    table, P = make_table(rng, [n], page)
    cache, tab = binding.kv_fp8_cache(P, 1, page, D), torch.from_numpy(table).cuda()
    k, v = (bf16(rng.standard_normal((1, 1, n, D))) for _ in range(2))
    v[0, 0, -1] = bf16(1.99 * 2.0 ** 127 * np.where(np.arange(D) % 3, 1.0, -1.0))
    binding.kv_fp8_write(cache, bf16_cuda(k), bf16_cuda(v), tab, whole([0]))
    q = bf16(rng.standard_normal((1, 4, Sq, D)))
    torch.cuda.synchronize()
    held = [host(t) for t in cache]
    want = attn_reference(q[:, :, :-1], held, table, [n - 1], None, True, 0, 0, D ** -0.5)
    for wg_rows in (16, 128):
        for splits in (1, 2):
            o, lse = call(q, held, table, [n], splits=splits, wg_rows=wg_rows)
            assert np.isinf(o[0, :, -1]).all() and (np.signbit(o[0, :, -1]) == (np.arange(D) % 3 == 0)).all()
            check((o[:, :, :-1], lse[:, :, :-1]), want, (wg_rows, splits))
