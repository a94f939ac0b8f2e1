"""The quantised cache on the GPU: written codes and exponents against the definition, bit for bit, and read back."""
import numpy as np
import pytest

from _kv_util import E4M3, bf16, bf16_cuda, gather_reference, host, make_cache, make_table, to_cuda, whole, write_reference

pytestmark = pytest.mark.gpu


def run_write(cache, table, k, v, start, count, layout="bhsd"):
    """kv_fp8_write on copies of the arrays, and the definition on others; both caches."""
    import torch
    from paper_2604_18616_amd import binding
    want = [t.copy() for t in cache]
    write_reference(want, k, v, table, start, count)
    dev, tab = to_cuda(cache, table)
    kd, vd = bf16_cuda(k), bf16_cuda(v)
    if layout == "bshd":
        kd, vd = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kd, vd))
    binding.kv_fp8_write(dev, kd, vd, tab, whole(start), whole(count))
    torch.cuda.synchronize()
    return [host(t) for t in dev], want


def check(got, want):
    for name, a, b in zip(("k", "v", "k_exp", "v_exp"), got, want):
        assert np.array_equal(a, b), (name, int((a != b).sum()), np.argwhere(a != b)[:4].tolist())


CASES = [
    # B, H, D, S, page, start, count
    (1, 1, 64, 1, 16, [0], None),
    (3, 2, 128, 1, 16, [0, 15, 37], None),                     # a new page, the last token of one, the middle
    (2, 4, 128, 5, 32, [30, 64], None),                        # over the end of a page
    (3, 3, 64, 130, 64, [0, 63, 129], [130, 1, 77]),
    (2, 2, 128, 300, 128, [0, 200], [299, 300]),
    (4, 1, 128, 40, 16, [3, 0, 16, 100], [0, 40, -5, 1000]),   # counts outside 0 ... S are the nearer end
    (1, 8, 64, 1000, 16, [7], None),
    (2, 3, 64, 100, 32, [17, 31], [100, 2]),
    (2, 2, 128, 150, 64, [5, 64], [150, 63]),
    (1, 3, 64, 260, 128, [127], None),
]


@pytest.mark.parametrize("B,H,D,S,page,start,count", CASES)
@pytest.mark.parametrize("layout", ["bhsd", "bshd"])
def test_written_codes_are_the_definitions(B, H, D, S, page, start, count, layout):
    rng = np.random.default_rng(B * 1000 + S)
    table, P = make_table(rng, [s + S for s in start], page)
    cache = make_cache(rng, P, H, page, D)
    # values of very different sizes from token to token: pages whose scale grows, and pages whose scale does not
    k, v = (bf16(rng.standard_normal((B, H, S, D)) * 2.0 ** rng.integers(-6, 7, (B, H, S, 1))) for _ in range(2))
    got, want = run_write(cache, table, k, v, start, count, layout)
    check(got, want)


@pytest.mark.parametrize("D,page", [(64, 16), (128, 128)])
def test_a_page_filled_token_by_token(D, page):
    """Each token twice the size of the one before: the scale grows with every call, and the codes are rounded again."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(5)
    table, P = make_table(rng, [page, page], page)
    cache = make_cache(rng, P, 2, page, D)
    want = [t.copy() for t in cache]
    dev, tab = to_cuda(cache, table)
    for t in range(12):
        k, v = (bf16(rng.standard_normal((2, 2, 1, D)) * 2.0 ** (t * s)) for s in (1, -1))
        write_reference(want, k, v, table, [t, t], None)
        binding.kv_fp8_write(dev, bf16_cuda(k), bf16_cuda(v), tab, whole([t, t]))
    torch.cuda.synchronize()
    check([host(t) for t in dev], want)


@pytest.mark.parametrize("page", [16, 64])
def test_values_at_the_borders(page):
    """Zeros, the largest and smallest numbers, ties, the largest value of a scale and the next one, NaN and infinities."""
    rng = np.random.default_rng(6)
    D, S = 64, 3 * page
    table, P = make_table(rng, [S], page)
    cache = make_cache(rng, P, 2, page, D)
    k, v = np.zeros((1, 2, S, D)), np.zeros((1, 2, S, D))
    k[0, 0, 0] = 448.0
    k[0, 0, 1] = -450.0                                        # (one bf16 step more: the next scale)
    k[0, 0, page:2 * page] = bf16(np.linspace(-2.0, 2.0, page * D).reshape(page, D) ** 9)
    k[0, 1, page - 1] = bf16(2.0 ** 127 * 1.99)
    k[0, 1, page] = 2.0 ** -126
    k[0, 1, 2 * page, :4] = [np.nan, np.inf, -np.inf, 3.0]
    v[0, 0, :page, 0] = [448.0 if t == 0 else (17 + t) / 16.0 for t in range(page)]       # ties of the rounding
    v[0, 0, page, :3] = [448.0, 2.0 ** -9, 2.0 ** -10]
    v[0, 0, page + 1, :4] = [3 * 2.0 ** -10, 2.0 ** -10 * 1.0078125, -2.0 ** -10, -0.0]
    v[0, 1] = np.nan
    got, want = run_write(cache, table, k, v, [0], None)
    check(got, want)


def test_missing_pages_and_positions_outside_the_table():
    rng = np.random.default_rng(7)
    page, D, S = 16, 64, 70
    table, P = np.array([[0, -1, 1, 2], [3, 4, 99, 5], [6, 7, 8, -7]], dtype=np.int32), 9
    cache = make_cache(rng, P, 2, page, D)
    k, v = (bf16(rng.standard_normal((3, 2, S, D))) for _ in range(2))
    got, want = run_write(cache, table, k, v, [0, -9, 2 ** 31 - 5], None)
    check(got, want)
    got, want = run_write(cache, table, k, v, [60, 3, -2 ** 31], [70, 70, 70])
    check(got, want)


@pytest.mark.parametrize("D,page,S,first", [(64, 16, 1, 0), (128, 16, 77, 0), (128, 64, 200, 0), (64, 128, 333, 100), (128, 32, 65, 31), (64, 64, 5, 900)])
def test_reading_back(D, page, S, first):
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(S)
    lens = [0, 1, 100, 290]
    table, P = make_table(rng, lens, page)
    if table.shape[1] > 2:
        table[3, 1] = -1
        table[2, 0] = P + 3
    cache = make_cache(rng, P, 3, page, D, spread=20)
    dev, tab = to_cuda(cache, table)
    k, v = binding.kv_fp8_read(dev, tab, whole(lens), S, first=first)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for h in range(3):
            wk, wv, there = gather_reference(cache, table, b, h, n)
            for got, ref in ((host(k)[b, h], wk), (host(v)[b, h], wv)):
                want = np.zeros((S, D))
                m = max(0, min(S, n - first))
                want[:m] = ref[first:first + m]
                assert np.array_equal(got, want), (b, h)


def test_every_code_and_exponent_is_read_exactly():
    """All codes at the largest, smallest and ordinary exponents (bf16 holds every one of them below 2^128), NaN as NaN."""
    import torch
    from paper_2604_18616_amd import binding
    exps = [27, 28, 100, 126, 127, 128, 200, 246, 247]
    P, page, D = len(exps), 16, 64
    codes = np.arange(256, dtype=np.uint8).repeat(4).reshape(page, D)
    cache = [np.broadcast_to(codes, (P, 1, page, D)).copy(), np.broadcast_to(codes.T, (P, 1, D, page)).copy()] + \
        [np.array(exps, dtype=np.uint8)[:, None] for _ in range(2)]
    dev, tab = to_cuda(cache, np.arange(P, dtype=np.int32)[None])
    k, v = binding.kv_fp8_read(dev, tab, whole([P * page]), P * page)
    torch.cuda.synchronize()
    want = bf16(np.clip(np.concatenate([E4M3[codes] * 2.0 ** (e - 127.0) for e in exps]), -2.0 ** 128, 2.0 ** 128))
    for got in (host(k)[0, 0], host(v)[0, 0]):
        assert np.array_equal(got, want, equal_nan=True)


def test_strided_rows_and_a_part_of_a_wider_table():
    """Keys and values as views of one projection's output, results read into views: nothing beside them is touched."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(8)
    B, H, D, S, page = 2, 3, 64, 37, 16
    table, P = make_table(rng, [S + 9] * B, page)
    cache = make_cache(rng, P, H, page, D)
    x = bf16(rng.standard_normal((B, S, 2 * H + 4, D)))
    buf = bf16_cuda(x)
    k, v = buf[:, :, 4:4 + H].transpose(1, 2), buf[:, :, 4 + H:].transpose(1, 2)
    xt = x.transpose(0, 2, 1, 3)
    want = [t.copy() for t in cache]
    write_reference(want, xt[:, 4:4 + H], xt[:, 4 + H:], table, [9, 0], [S, 20])
    dev, tab = to_cuda(cache, table)
    wide = torch.full((B, table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + table.shape[1]] = tab
    part = wide[:, 2:2 + table.shape[1]]
    assert binding.kv_fp8_write(dev, k, v, part, whole([9, 0]), whole([S, 20])) is dev
    torch.cuda.synchronize()
    check([host(t) for t in dev], want)
    room = torch.full((B, S + 2, 2 * H, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = (room[:, 1:1 + S, h:h + H, :D].transpose(1, 2) for h in (0, H))
    got = binding.kv_fp8_read(dev, part, whole([S + 9, 20]), S, first=3, k=ko, v=vo)
    torch.cuda.synchronize()
    assert got[0] is ko and got[1] is vo
    for b, n in enumerate((S + 9, 20)):
        for h in range(H):
            for out, ref in zip((host(ko)[b, h], host(vo)[b, h]), gather_reference(want, table, b, h, n)):
                m = min(S, n - 3)
                assert np.array_equal(out[:m], ref[3:3 + m]) and not out[m:].any()
    ko.fill_(7.0), vo.fill_(7.0)
    assert (room == 7.0).all()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("S", [1, 16, 17, 90])
def test_a_start_inside_a_missing_page(page, S):
    """The first new tokens would lie behind others of a page that is not there; every start in a page, few tokens and more."""
    rng = np.random.default_rng(page + S)
    D, starts = 64, [page + 5, 7, 2 * page - 1, page - 4, 3]
    table, P = make_table(rng, [s + S for s in starts], page)
    table[0, 1], table[1, 0], table[2, 1] = -1, P, 2 ** 31 - 1
    cache = make_cache(rng, P, 2, page, D)
    k, v = (bf16(rng.standard_normal((len(starts), 2, S, D)) * 2.0 ** rng.integers(-6, 7, (len(starts), 2, S, 1))) for _ in range(2))
    check(*run_write(cache, table, k, v, starts, None))


@pytest.mark.parametrize("D,page", [(64, 16), (128, 16), (128, 128), (64, 64)])
@pytest.mark.parametrize("S,first", [(1, 0), (1, 31), (3, 15), (16, 0), (16, 1), (16, 47), (7, 64), (17, 15), (5, 2 ** 31 - 1)])
def test_reading_a_few_positions(D, page, S, first):
    """Up to 16 positions, which may lie in two pages of which one is missing, before, across and behind a sequence's end."""
    import torch
    from paper_2604_18616_amd import binding
    rng = np.random.default_rng(S + page)
    lens = [0, 1, 16, 33, 50, 64, 200]
    table, P = make_table(rng, lens, page)
    if table.shape[1] > 2:
        table[3, 1], table[5, 2], table[6, 3] = -1, P, -7
    cache = make_cache(rng, P, 3, page, D, spread=20)
    dev, tab = to_cuda(cache, table)
    room = torch.full((len(lens), S, 6, D), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = (room[:, :, h:h + 3].transpose(1, 2) for h in (0, 3))
    binding.kv_fp8_read(dev, tab, whole(lens), S, first=first, k=k, v=v)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for h in range(3):
            wk, wv, _ = gather_reference(cache, table, b, h, n)
            for got, ref in ((host(k)[b, h], wk), (host(v)[b, h], wv)):
                want = np.zeros((S, D))
                m = max(0, min(S, n - first))
                want[:m] = ref[first:first + m]
                assert np.array_equal(got, want), (b, h)
