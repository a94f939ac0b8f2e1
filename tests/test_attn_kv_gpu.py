"""Attention over the quantised cache against its definition in 64 bits."""
import numpy as np
import pytest

from _kv_util import attn_reference, bf16, bf16_cuda, host, make_cache, make_table, quantise, spoil_behind, to_cuda, whole

pytestmark = pytest.mark.gpu


def run(q, cache, table, lens, q_lens=None, causal=True, window=0, sinks=0, scale=None, layout="bhsd", **more):
    import torch
    from paper_2604_18616_amd import binding
    dev, tab = to_cuda(cache, table)
    qd = bf16_cuda(q)
    if layout == "bshd":
        qd = qd.transpose(1, 2).contiguous().transpose(1, 2)
    o = torch.full_like(qd, float("nan"))
    lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda")
    binding.attn_kv_fp8(qd, dev, tab, whole(lens), whole(q_lens), o=o, lse=lse, causal=causal, window=window, sinks=sinks, scale=scale, **more)
    torch.cuda.synchronize()
    return host(o), host(lse).astype(np.float64)


def check(got, want):
    (o, lse), (wo, wl, to, tl) = got, want
    gone = np.isneginf(wl)
    assert np.array_equal(np.isneginf(lse), gone)
    assert np.all(np.abs(lse[~gone] - wl[~gone]) <= tl[~gone]), np.abs(lse[~gone] - wl[~gone]).max()
    assert np.all(np.abs(o - wo) <= to), (float((np.abs(o - wo) - to).max()), np.argwhere(~(np.abs(o - wo) <= to))[:4].tolist())
    assert not o[gone].any()


def case(seed, B, Hq, Hkv, D, Sq, lens, page, **kw):
    rng = np.random.default_rng(seed)
    table, P = make_table(rng, lens, page, width=kw.pop("width", None))
    cache = make_cache(rng, P, Hkv, page, D)
    spoil_behind(cache, table, lens)
    q = bf16(rng.standard_normal((B, Hq, Sq, D)) * kw.pop("size", 1.0))
    layout = kw.pop("layout", "bhsd")
    scale = kw.get("scale") or D ** -0.5
    want = attn_reference(q, cache, table, lens, kw.get("q_lens"), kw.get("causal", True), kw.get("window", 0), kw.get("sinks", 0), scale)
    for wg_rows in (0, 16, 128):
        print("wg_rows", wg_rows, flush=True)
        check(run(q, cache, table, lens, layout=layout, wg_rows=wg_rows, **kw), want)


SHAPES = [
    # B, Hq, Hkv, D, Sq, lens, page
    (1, 1, 1, 64, 1, [1], 16),
    (1, 1, 1, 128, 1, [1], 128),
    (3, 4, 2, 128, 1, [0, 64, 65], 16),
    (4, 8, 1, 64, 1, [63, 128, 129, 700], 32),
    (2, 16, 2, 128, 1, [1000, 15], 64),
    (2, 5, 1, 128, 2, [300, 2], 128),
    (1, 32, 8, 128, 1, [2000], 16),
    (2, 6, 2, 64, 7, [200, 5], 64),               # fewer keys than query rows
    (1, 12, 4, 128, 17, [333], 32),
    (2, 4, 4, 64, 33, [257, 40], 16),
    (1, 16, 1, 128, 9, [515], 16),
    (2, 4, 2, 128, 130, [400, 131], 64),
    (1, 3, 1, 64, 200, [777], 128),
    (1, 2, 2, 128, 100, [100], 16),
]


@pytest.mark.parametrize("B,Hq,Hkv,D,Sq,lens,page", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_against_the_definition(B, Hq, Hkv, D, Sq, lens, page, causal):
    case(Sq + 7 * Hq, B, Hq, Hkv, D, Sq, lens, page, causal=causal, layout="bshd" if causal else "bhsd")


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 64), (100, 70), (127, 3), (4000, 4), (65, 2 ** 31 - 1)])
@pytest.mark.parametrize("B,Hq,Hkv,D,Sq,lens,page", [(3, 4, 2, 128, 1, [500, 90, 3], 16), (2, 4, 1, 64, 5, [700, 64], 32), (1, 4, 2, 128, 90, [430], 64)])
def test_windows_and_sinks(B, Hq, Hkv, D, Sq, lens, page, window, sinks):
    case(window, B, Hq, Hkv, D, Sq, lens, page, window=window, sinks=sinks)
    case(window + 1, B, Hq, Hkv, D, Sq, lens, page, window=window, sinks=sinks, causal=False)


@pytest.mark.parametrize("B,Hq,Hkv,D,Sq,lens,page", [(4, 4, 2, 128, 6, [300, 40, 6, 0], 16), (3, 8, 2, 64, 50, [300, 90, 50], 64), (3, 4, 4, 128, 150, [300, 190, 149], 32)])
def test_fewer_query_rows_for_some(B, Hq, Hkv, D, Sq, lens, page):
    case(3, B, Hq, Hkv, D, Sq, lens, page, q_lens=[Sq, 1, 0, -3][:B])
    case(4, B, Hq, Hkv, D, Sq, lens, page, q_lens=[Sq + 9, Sq // 2, 2, 1][:B], window=20, sinks=2)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 40, 256])
@pytest.mark.parametrize("B,Hq,Hkv,D,Sq,lens", [(2, 8, 2, 128, 1, [900, 70]), (1, 4, 2, 64, 20, [650]), (1, 4, 1, 128, 100, [700])])
def test_cut_keys(B, Hq, Hkv, D, Sq, lens, splits):
    """Every number of parts, also more than there are tiles, through the C entry point with the caller's memory."""
    import ctypes
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(splits)
    page = 32
    table, P = make_table(rng, lens, page)
    cache = make_cache(rng, P, Hkv, page, D)
    spoil_behind(cache, table, lens)
    q = bf16(rng.standard_normal((B, Hq, Sq, D)))
    dev, tab = to_cuda(cache, table)
    struct = binding._cache_struct(dev)[0]
    lib, qd = binding.load_library(), bf16_cuda(q)
    o, lse = torch.full_like(qd, float("nan")), torch.full((B, Hq, Sq), float("nan"), dtype=torch.float32, device="cuda")
    need = 4 * B * Hq * Sq * splits * (D + 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    st = (ctypes.c_longlong * 3)(*qd.stride()[:3])
    print("splits", splits, lens, flush=True)
    dl = whole(lens)
    want = attn_reference(q, cache, table, lens, None, True, 0, 0, D ** -0.5)
    for wg_rows in (0, 16, 128):
        o.fill_(float("nan")), lse.fill_(float("nan")), ws.fill_(0xFF)
        rc = lib.attn_kv_fp8(qd.data_ptr(), ctypes.byref(struct), tab.data_ptr(), tab.stride(0), tab.shape[1], dl.data_ptr(), None, o.data_ptr(), lse.data_ptr(),
                             B, Hq, Sq, st, st, 1, 0, 0, D ** -0.5, 0, ws.data_ptr(), need, splits, wg_rows, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()
        check((host(o), host(lse).astype(np.float64)), want)


def test_large_scores_and_scales():
    case(11, 2, 4, 2, 128, 3, [400, 77], 16, size=30.0)                     # nearly one key per row counts
    case(12, 2, 4, 2, 64, 40, [400, 77], 64, scale=3.0)
    case(13, 1, 4, 2, 64, 3, [300], 64, scale=1e-6)                         # all keys count the same


def test_missing_pages_are_not_seen():
    rng = np.random.default_rng(21)
    for Sq, page in ((1, 16), (1, 64), (30, 32), (140, 128)):
        lens = [600, 300, 500]
        table, P = make_table(rng, lens, page)
        table[0, 0] = -1
        table[0, 2] = P                              # not a page
        table[1, :] = -2 ** 31                       # nothing at all
        table[2, -1] = 2 ** 31 - 1
        cache = make_cache(rng, P, 2, page, 64)
        q = bf16(rng.standard_normal((3, 4, Sq, 64)))
        want = attn_reference(q, cache, table, lens, None, True, 0, 0, 0.125)
        for wg_rows in (16, 128):
            check(run(q, cache, table, lens, wg_rows=wg_rows), want)


def test_lengths_outside_the_table_and_max_len():
    rng = np.random.default_rng(22)
    table, P = make_table(rng, [128, 100], 16)
    cache = make_cache(rng, P, 2, 16, 128)
    q = bf16(rng.standard_normal((2, 4, 2, 128)))
    for lens, limit, taken in (([10 ** 9, -5], 0, [128, 0]), ([128, 100], 90, [90, 90])):
        want = attn_reference(q, cache, table, taken, None, True, 0, 0, 128 ** -0.5)
        for wg_rows in (16, 128):
            check(run(q, cache, table, lens, max_len=limit, wg_rows=wg_rows), want)


@pytest.mark.parametrize("Sq,D,window", [(4, 128, 0), (4, 64, 30), (70, 128, 0), (200, 64, 40)])
@pytest.mark.parametrize("wg_rows", [16, 128])
def test_nan_reaches_the_rows_that_see_it(Sq, D, window, wg_rows):
    """NaN codes in V and in K among the last tokens and at a window's end: rows before them and past them stay finite."""
    rng = np.random.default_rng(Sq)
    lens, page = [Sq + 90], 16
    table, P = make_table(rng, lens, page)
    cache = make_cache(rng, P, 1, page, D)
    q = bf16(rng.standard_normal((1, 2, Sq, D)))
    for which, pos, d in ((1, lens[0] - 2, 5), (1, lens[0] - Sq, D - 1), (0, lens[0] - 3, 0), (1, 70, 9)):
        spoilt = [t.copy() for t in cache]
        at = table[0, pos // page]
        if which:
            spoilt[1][at, 0, d, pos % page] = 0xFF
        else:
            spoilt[0][at, 0, pos % page, d] = 0x7F
        o, lse = run(q, spoilt, table, lens, window=window, wg_rows=wg_rows)
        wo, wl, to, tl = attn_reference(q, cache, table, lens, None, True, window, 0, D ** -0.5)
        row_pos = lens[0] - Sq + np.arange(Sq)
        sees = (pos <= row_pos) & ((pos > row_pos - window) if window else True)
        assert sees.any() and (not sees.all() or pos <= row_pos[0])
        if which:
            assert np.isnan(o[0, :, sees, d]).all()
            o[0][:, sees, d] = wo[0][:, sees, d]
        else:
            assert np.isnan(o[0][:, sees]).all() and np.isnan(lse[0][:, sees]).all()
            o[0][:, sees], lse[0][:, sees] = wo[0][:, sees], wl[0][:, sees]
        check((o, lse), (wo, wl, to, tl))


def test_a_page_shared_by_two_sequences():
    rng = np.random.default_rng(31)
    table = np.array([[0, 1, 2], [0, 1, 3]], dtype=np.int32)
    cache = make_cache(rng, 4, 2, 16, 64)
    q = bf16(rng.standard_normal((2, 4, 1, 64)))
    want = attn_reference(q, cache, table, [40, 47], None, False, 0, 0, 0.125)
    check(run(q, cache, table, [40, 47], causal=False), want)


@pytest.mark.parametrize("Hq,Sq", [(17, 1), (3, 11), (64, 1), (7, 19), (1, 257), (40, 13)])
@pytest.mark.parametrize("D", [64, 128])
def test_odd_numbers_of_packed_rows(Hq, Sq, D):
    """From just over one block of rows to more than four blocks of the other kind; a workgroup's last rows are none."""
    case(Hq * Sq + D, 1, Hq, 1, D, Sq, [Sq + 150], 32, layout="bshd")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ramp", [0.5, 4.0, -4.0, 40.0])
def test_scores_that_rise_along_the_cache(D, ramp):
    """Every tile's largest score exceeds the one before by a little, by much, or not at all: the maximum that the
    probabilities are taken relative to is made anew now and then, always and never."""
    rng = np.random.default_rng(int(abs(ramp) * 2) + D)
    lens, page = [1500, 900], 64
    table, P = make_table(rng, lens, page)
    cache = make_cache(rng, P, 1, page, D)
    cache[2][:] = 127 - 7
    for b, n in enumerate(lens):
        for slot in range(-(-n // page)):
            value = ramp * (slot - n // page // 2)           # of column 0: an exact code's, whose page's exponent is 0
            cache[0][table[b, slot], 0, :, 0] = quantise(np.clip(value, -3.5, 3.5) * 128, 0)
    spoil_behind(cache, table, lens)
    for Sq in (1, 40):
        q = bf16(rng.standard_normal((2, 4, Sq, D)) * 0.1)
        q[..., 0] = 16.0
        want = attn_reference(q, cache, table, lens, None, True, 0, 0, 1.0)
        for wg_rows in (16, 128):
            check(run(q, cache, table, lens, scale=1.0, wg_rows=wg_rows), want)


@pytest.mark.parametrize("Sq", [3, 60])
@pytest.mark.parametrize("wg_rows", [16, 128])
def test_padded_rows_of_q_may_hold_anything(Sq, wg_rows):
    rng = np.random.default_rng(41)
    lens, q_lens = [200, 300, 90], [Sq, Sq - 2, 0]
    table, P = make_table(rng, lens, 16)
    cache = make_cache(rng, P, 2, 16, 64)
    q = bf16(rng.standard_normal((3, 4, Sq, 64)))
    want = attn_reference(q, cache, table, lens, q_lens, True, 0, 0, 0.125)
    for b, n in enumerate(q_lens):
        q[b, :, n:] = np.nan
    check(run(q, cache, table, lens, q_lens=q_lens, wg_rows=wg_rows), want)


def test_more_sequences_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(42)
    lens = [int(n) for n in rng.integers(0, 260, 150)]
    lens[149] = 2000                                         # the longest one, by which all are cut, is the last
    table, P = make_table(rng, lens, 16)
    cache = make_cache(rng, P, 1, 16, 64)
    spoil_behind(cache, table, lens)
    for Sq in (1, 20):
        q = bf16(rng.standard_normal((150, 2, Sq, 64)))
        want = attn_reference(q, cache, table, lens, None, True, 0, 0, 0.125)
        for wg_rows in (0, 16, 128):
            check(run(q, cache, table, lens, wg_rows=wg_rows), want)


@pytest.mark.parametrize("Sq", [1, 50])
def test_views(Sq):
    """Exponents at odd addresses, a page table that is a part of a wider one, q and o with heads and rows apart, o given."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(43)
    lens, D, page = [333, 250], 128, 32
    table, P = make_table(rng, lens, page)
    cache = make_cache(rng, P, 3, page, D)
    q = bf16(rng.standard_normal((2, 6, Sq, D)))
    dev, tab = to_cuda(cache, table)
    odd = []
    for t, skip in ((dev.k_exp, 1), (dev.v_exp, 3)):
        room = torch.full((t.numel() + 8,), 255, dtype=torch.uint8, device="cuda")
        odd.append(room[skip:skip + t.numel()].view(t.shape))
        odd[-1].copy_(t)
    dev = binding.KvFp8Cache(dev.k, dev.v, *odd)
    wide = torch.full((2, table.shape[1] + 7), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + table.shape[1]] = tab
    room = torch.full((2, Sq, 9, D + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    qd = room[:, :, 1:7, :D].transpose(1, 2)
    qd.copy_(bf16_cuda(q))
    want = attn_reference(q, cache, table, lens, None, True, 0, 0, D ** -0.5)
    for wg_rows in (0, 16, 128):
        out = torch.full((2, 7, Sq + 3, 2 * D), 7.0, dtype=torch.bfloat16, device="cuda")
        o = out[:, 1:, 1:1 + Sq, D:]
        got = binding.attn_kv_fp8(qd, dev, wide[:, 3:3 + table.shape[1]], whole(lens), o=o, causal=True, wg_rows=wg_rows)
        torch.cuda.synchronize()
        assert got[0] is o
        check((host(o), host(got[1]).astype(np.float64)), want)
        o.fill_(7.0)
        assert (out == 7.0).all()                            # nothing beside o was written


def test_the_librarys_own_cut_is_the_same_call():
    """Letting the library cut, and asking for the cut that its workspace is made for: the same bits."""
    import ctypes
    import torch
    from paper_2604_18616_amd import binding
    lib, seen = binding.load_library(), set()
    for B, Hq, Hkv, D, Sq, longest in ((1, 8, 8, 64, 1, 300), (1, 8, 1, 128, 1, 5000), (3, 4, 2, 64, 4, 3500), (1, 4, 1, 128, 20, 9000), (1, 2, 1, 64, 300, 6000), (2, 8, 2, 128, 1, 200)):
        rng = np.random.default_rng(longest)
        table, P = make_table(rng, [longest] * B, 64)
        dev, tab = to_cuda(make_cache(rng, P, Hkv, 64, D), table)
        qd = bf16_cuda(bf16(rng.standard_normal((B, Hq, Sq, D))))
        need = lib.attn_kv_fp8_workspace_bytes(B, Hq, Hkv, Sq, longest, D, 0, 0)
        splits = need // (4 * B * Hq * Sq * (D + 2))
        seen.add(splits)
        struct, lens = binding._cache_struct(dev)[0], whole([longest] * B)
        ws, st, results = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), (ctypes.c_longlong * 3)(*qd.stride()[:3]), []
        for cut in (0, max(splits, 1)):
            o, lse = torch.full_like(qd, float("nan")), torch.full((B, Hq, Sq), float("nan"), device="cuda")
            rc = lib.attn_kv_fp8(qd.data_ptr(), ctypes.byref(struct), tab.data_ptr(), tab.stride(0), tab.shape[1], lens.data_ptr(), None, o.data_ptr(), lse.data_ptr(),
                                 B, Hq, Sq, st, st, 1, 0, 0, 0.1, longest, ws.data_ptr(), need, cut, 0, torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            torch.cuda.synchronize()
            results.append((o, lse))
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
        assert not torch.isnan(results[0][0]).any()
    assert len(seen) > 2


def test_two_calls_at_once():
    """Two streams, each call with memory of its own for its parts: the bits of the calls one after the other."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(44)
    lens, D = [9000], 128
    table, P = make_table(rng, lens, 64)
    dev, tab = to_cuda(make_cache(rng, P, 2, 64, D), table)
    dl, sides = whole(lens), [torch.cuda.Stream() for _ in range(2)]
    qs = [bf16_cuda(bf16(rng.standard_normal((1, 8, Sq, D)))) for Sq in (1, 60)]
    want = [binding.attn_kv_fp8(q, dev, tab, dl, causal=True) for q in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[i].append(binding.attn_kv_fp8(qs[i], dev, tab, dl, causal=True))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])


@pytest.mark.parametrize("D,window,Sq", [(64, 0, 1), (128, 0, 1), (64, 30, 2), (128, 9, 5)])
def test_many_short_sequences(D, window, Sq):
    """Where a wavefront by itself takes a sequence's head: 0 to 130 keys, some pages missing, NaN behind the ends."""
    rng = np.random.default_rng(D + window)
    lens = [int(n) for n in rng.integers(0, 131, 200)]
    table, P = make_table(rng, lens, 16)
    table[rng.random(table.shape) < 0.05] = -1
    cache = make_cache(rng, P, 2, 16, D)
    spoil_behind(cache, table, lens)
    q = bf16(rng.standard_normal((200, 6, Sq, D)))
    want = attn_reference(q, cache, table, lens, None, True, window, 2 if window else 0, D ** -0.5)
    for limit in (0, 131):
        check(run(q, cache, table, lens, window=window, sinks=2 if window else 0, max_len=limit), want)


@pytest.mark.parametrize("D,window,Sq", [(64, 0, 1), (128, 0, 1), (128, 70, 2)])
def test_a_batch_with_a_few_long_sequences(D, window, Sq):
    """Where eight wavefronts share a sequence's head: 32 sequences, some with 1500 keys, most with few, some with none."""
    rng = np.random.default_rng(D + Sq)
    lens = [1500, 1337, 1024] + [int(n) for n in rng.integers(0, 160, 29)]
    table, P = make_table(rng, lens, 16)
    table[0, 3], table[1, 80] = -1, P
    cache = make_cache(rng, P, 8, 16, D)
    spoil_behind(cache, table, lens)
    q = bf16(rng.standard_normal((32, 16, Sq, D)))
    want = attn_reference(q, cache, table, lens, None, True, window, 3 if window else 0, D ** -0.5)
    check(run(q, cache, table, lens, window=window, sinks=3 if window else 0), want)
