"""The operators of the quantised cache together, as a program that serves uses them: prompts in chunks, then token by token;
through the extension module and without it, captured and replayed, on another stream."""
import numpy as np
import pytest

from _kv_util import attn_reference, bf16, host, make_table, write_reference

pytestmark = pytest.mark.gpu


def modes():
    """The binding with the extension module and without it."""
    from paper_2604_18616_amd import binding
    for native in (None, False):
        binding._native = native
        yield native
    binding._native = None


@pytest.fixture(autouse=True)
def restore():
    yield
    from paper_2604_18616_amd import binding
    binding._native = None


def same(a, b):
    import torch
    as_int = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])
    return a.shape == b.shape and a.stride() == b.stride() and a.dtype == b.dtype and torch.equal(as_int(a), as_int(b))


class Layer:
    """One attention layer's heads, positions and cache on the GPU, and what the cache has to hold on the host."""

    def __init__(self, seed, B, Hq, Hkv, D, page, most):
        import torch
        from paper_2604_18616_amd import binding
        self.rng = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.D, self.page = B, Hq, Hkv, D, page
        self.table, self.P = make_table(self.rng, [most] * B, page)
        self.tab = torch.from_numpy(self.table).cuda()
        self.cache = binding.kv_fp8_cache(self.P, Hkv, page, D)
        for t in self.cache:
            t.fill_(0x7F)                                    # what memory holds before it is written: here NaN
        self.inv = binding.rope_frequencies(D, factor=4.0, original_len=4096)

    def fresh(self, S):
        """A projection's output, q, k and v side by side."""
        import torch
        x = bf16(self.rng.standard_normal((self.B, S, self.Hq + 2 * self.Hkv, self.D)))
        return torch.from_numpy(x).to(torch.bfloat16).cuda()

    def step(self, x, start, count, window=0, sinks=0):
        """q and k turned where they lie, k and v appended, attention over what the cache holds then."""
        import torch
        from paper_2604_18616_amd import binding
        q, k, v = (t.transpose(1, 2) for t in x.split((self.Hq, self.Hkv, self.Hkv), 2))
        positions = start[:, None] + torch.arange(x.shape[1], dtype=torch.int32, device="cuda")
        q, k = binding.rope_bf16(q, positions, self.inv, k=k)
        binding.kv_fp8_write(self.cache, k, v, self.tab, start, count=count)
        lens = start + (x.shape[1] if count is None else count)
        return q, k, v, binding.attn_kv_fp8(q, self.cache, self.tab, lens, q_lens=count, causal=True, window=window, sinks=sinks)


@pytest.mark.parametrize("B,Hq,Hkv,D,page,window,sinks", [(2, 4, 2, 128, 16, 0, 0), (3, 8, 1, 64, 64, 40, 3)])
def test_prompts_in_chunks_then_tokens(B, Hq, Hkv, D, page, window, sinks):
    import torch
    layer = Layer(1, B, Hq, Hkv, D, page, 300)
    want = [host(t) for t in layer.cache]
    held = np.zeros(B, dtype=np.int64)
    for S, counts in ((70, [70, 41, 1][:B]), (64, [1, 64, 0][:B]), (1, None), (1, None), (3, [3, 0, 2][:B]), (150, None), (1, None)):
        start = torch.tensor(held.tolist(), dtype=torch.int32, device="cuda")
        count = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        q, k, v, (o, lse) = layer.step(layer.fresh(S), start, count, window, sinks)
        torch.cuda.synchronize()
        write_reference(want, host(k), host(v), layer.table, held, counts)
        for a, b in zip(layer.cache, want):
            assert np.array_equal(host(a), b)
        lens = held + (S if counts is None else np.array(counts))
        wo, wl, to, tl = attn_reference(host(q), want, layer.table, lens, counts, True, window, sinks, D ** -0.5)
        gone = np.isneginf(wl)
        assert np.array_equal(np.isneginf(host(lse)), gone) and np.all(np.abs(host(lse)[~gone] - wl[~gone]) <= tl[~gone])
        assert np.all(np.abs(host(o) - wo) <= to) and not host(o)[gone].any()
        held = lens


@pytest.mark.parametrize("Sq,count", [(1, None), (5, [5, 2]), (90, [30, 90])])
def test_with_the_extension_module_and_without(Sq, count):
    """The same bits and the same memory formats both ways."""
    import torch
    from paper_2604_18616_amd import binding
    results = []
    for _ in modes():
        layer = Layer(2, 2, 8, 2, 128, 32, 400)
        start = torch.tensor([200, 131], dtype=torch.int32, device="cuda")
        x = layer.fresh(300)
        layer.step(x, torch.zeros_like(start), None)
        counts = None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda")
        q, k, v, (o, lse) = layer.step(layer.fresh(Sq), start, counts)
        rk, rv = binding.kv_fp8_read(layer.cache, layer.tab, start, 77, first=60)
        plain_q = binding.rope_bf16(x.transpose(1, 2), torch.arange(300, dtype=torch.int32, device="cuda"), layer.inv, interleaved=True, inverse=True, scale=0.5)
        none = binding.attn_kv_fp8(q, layer.cache, layer.tab, start, max_len=100, scale=0.3)
        results.append((q, k, o, lse, rk, rv, plain_q, *none, *layer.cache))
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert same(a, b)


def test_refusals_both_ways():
    import torch
    from paper_2604_18616_amd import binding
    layer = Layer(3, 2, 4, 2, 64, 16, 64)
    c, t = layer.cache, layer.tab
    x = torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    pos, inv = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), layer.inv
    K = binding.KvFp8Cache
    calls = [
        lambda: binding.kv_fp8_write(c, x.float(), x, t, n), lambda: binding.kv_fp8_write(c, x[:1], x, t, n), lambda: binding.kv_fp8_write(c, x, x[:, :, :2], t, n),
        lambda: binding.kv_fp8_write(c, x, x, t.long(), n), lambda: binding.kv_fp8_write(c, x, x, t[:1], n), lambda: binding.kv_fp8_write(c, x, x, t, n.long()),
        lambda: binding.kv_fp8_write(c, x, x, t, n[:1]), lambda: binding.kv_fp8_write(c, x, x, t, None), lambda: binding.kv_fp8_write(c, x, x, t, n, count=n.cpu()),
        lambda: binding.kv_fp8_write(K(c.k, c.k, c.k_exp, c.v_exp), x, x, t, n), lambda: binding.kv_fp8_write(K(c.k[:1], c.v, c.k_exp, c.v_exp), x, x, t, n),
        lambda: binding.kv_fp8_write(K(c.k.float(), c.v, c.k_exp, c.v_exp), x, x, t, n), lambda: binding.kv_fp8_write(K(c.k.cpu(), c.v, c.k_exp, c.v_exp), x, x, t, n),
        lambda: binding.kv_fp8_write(c, x[:, :, :0], x[:, :, :0], t, n), lambda: binding.kv_fp8_write(c, x[:, :, :1].expand(2, 2, 3, 64), x, t, n),
        lambda: binding.kv_fp8_read(c, t, n, 0), lambda: binding.kv_fp8_read(c, t, n, 4, first=-1), lambda: binding.kv_fp8_read(c, t.cpu(), n, 4),
        lambda: binding.attn_kv_fp8(q[:, :3], c, t, n), lambda: binding.attn_kv_fp8(q.half(), c, t, n), lambda: binding.attn_kv_fp8(q, c, t, n, q_lens=n[:1]),
        lambda: binding.attn_kv_fp8(q, c, t, n, window=-1), lambda: binding.attn_kv_fp8(q, c, t, n, sinks=-2), lambda: binding.attn_kv_fp8(q, c, t, n, scale=-1.0),
        lambda: binding.attn_kv_fp8(q, c, t, n, max_len=-1), lambda: binding.attn_kv_fp8(q, c, t, n, scale=float("nan")), lambda: binding.attn_kv_fp8(q[0], c, t, n),
        lambda: binding.attn_kv_fp8(q[..., ::2], c, t, n), lambda: binding.attn_kv_fp8(q.cpu(), c, t, n), lambda: binding.attn_kv_fp8(q, c, t[:, :0], n),
        lambda: binding.rope_bf16(q, pos[:1], inv), lambda: binding.rope_bf16(q, pos.long(), inv), lambda: binding.rope_bf16(q, pos, inv.float()),
        lambda: binding.rope_bf16(q, pos, torch.ones(40, dtype=torch.float64, device="cuda")), lambda: binding.rope_bf16(q, pos, inv[:0]),
        lambda: binding.rope_bf16(q, pos, inv, k=x[:, :, :2]), lambda: binding.rope_bf16(q, pos, inv, scale=float("inf")), lambda: binding.rope_bf16(q, pos.cpu(), inv),
        lambda: binding.rope_bf16(q, pos, inv, k_out=x), lambda: binding.rope_bf16(q[..., 1:61], pos, inv[:30]),
    ]
    for i, call in enumerate(calls):
        said = []
        for _ in modes():
            with pytest.raises(Exception) as e:
                call()
            said.append((type(e.value), str(e.value)))
        assert said[0] == said[1] and said[0][0] in (ValueError, binding.AttnError), (i, said)


@pytest.mark.parametrize("Sq", [1, 4, 40, 200])
def test_captured_steps_replay_to_the_eager_bits(Sq):
    """Two graphs, captured one after the other, replayed in turn with eager work between: each into its own outputs, the
    lengths and tables read when it runs."""
    import torch
    from paper_2604_18616_amd import binding
    eager, captured = Layer(4, 2, 8, 2, 128, 16, 700), Layer(4, 2, 8, 2, 128, 16, 700)
    first = eager.fresh(300)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    for layer in (eager, captured):
        layer.step(first.clone(), zero, None)
    torch.cuda.synchronize()
    start, x = torch.full((2,), 300, dtype=torch.int32, device="cuda"), eager.fresh(Sq)
    graphs = []
    snapshot = [t.clone() for t in captured.cache]
    captured.step(x, start, None)                            # (warm-up)
    for t, s in zip(captured.cache, snapshot):
        t.copy_(s)
    torch.cuda.synchronize()
    for window in (0, 50):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = captured.step(x, start, None, window, 2 if window else 0)
        graphs.append((graph, out, window))
    for turn in range(3):
        start.copy_(torch.tensor([300 + turn, 290 - turn], dtype=torch.int32))
        x.copy_(eager.fresh(Sq))
        for graph, out, window in graphs:
            graph.replay()
            want = eager.step(x, start, None, window, 2 if window else 0)
            scratch = torch.randn(1 << 20, device="cuda").sum()
            torch.cuda.synchronize()
            for a, b in zip((out[0], out[1], *out[3], *captured.cache), (want[0], want[1], *want[3], *eager.cache)):
                assert same(a, b), (turn, window)
            assert torch.isfinite(scratch)


def test_on_another_stream():
    import torch
    from paper_2604_18616_amd import binding
    layer = Layer(5, 2, 8, 2, 128, 32, 2000)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    q = layer.step(layer.fresh(1500), zero, None)[0][:, :, -1:].contiguous()
    lens = torch.full((2,), 1500, dtype=torch.int32, device="cuda")
    want = binding.attn_kv_fp8(q, layer.cache, layer.tab, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                            # torch's current stream: the keys are cut there too
        got = binding.attn_kv_fp8(q, layer.cache, layer.tab, lens)
    o, lse = torch.empty_like(q), torch.empty((2, 8, 1), device="cuda")
    side.synchronize()
    binding.attn_kv_fp8(q, layer.cache, layer.tab, lens, o=o, lse=lse, stream=side)     # not torch's: uncut
    side.synchronize()
    assert same(got[0], want[0]) and same(got[1], want[1])
    assert (o.float() - want[0].float()).abs().max() <= 2.0 ** -7 * want[0].float().abs().max() and (lse - want[1]).abs().max() <= 1e-5


def test_the_same_bits_every_time():
    import torch
    from paper_2604_18616_amd import binding
    layer = Layer(6, 3, 16, 2, 64, 64, 5000)
    layer.step(layer.fresh(4000), torch.zeros(3, dtype=torch.int32, device="cuda"), None)
    lens = torch.tensor([4000, 77, 2500], dtype=torch.int32, device="cuda")
    for Sq in (1, 16, 100):
        q = layer.fresh(Sq)[:, :, :16].transpose(1, 2)
        results = [binding.attn_kv_fp8(q, layer.cache, layer.tab, lens, causal=True) for _ in range(4)]
        torch.cuda.synchronize()
        for o, lse in results[1:]:
            assert same(o, results[0][0]) and same(lse, results[0][1])


@pytest.mark.parametrize("Sq", [1, 150])
def test_offsets_past_32_bits(Sq):
    """Pages behind the first 4 GiB of codes: written, attended to and read back as in a small cache."""
    import torch
    from paper_2604_18616_amd import binding
    page, D, H, far = 128, 128, 2, 1 << 17                   # far * H * page * D = 2^32
    rng = np.random.default_rng(9)
    order = rng.permutation(8)
    near_table = torch.from_numpy(order.reshape(2, 4).astype(np.int32)).cuda()
    near, large = binding.kv_fp8_cache(8, H, page, D), binding.kv_fp8_cache(far + 8, H, page, D)
    for t in near:
        t.fill_(0x7F)
    for t in large:
        t[far:].fill_(0x7F)
    x = torch.from_numpy(bf16(rng.standard_normal((2, 450, H, D)))).to(torch.bfloat16).cuda().transpose(1, 2)
    q = torch.from_numpy(bf16(rng.standard_normal((2, 8, Sq, D)))).to(torch.bfloat16).cuda()
    lens = torch.tensor([451, 463], dtype=torch.int32, device="cuda")
    results = []
    for cache, table in ((near, near_table), (large, near_table + far)):
        binding.kv_fp8_write(cache, x, 2 * x, table, torch.tensor([1, 13], dtype=torch.int32, device="cuda"))
        binding.kv_fp8_write(cache, -x[:, :, :20], x[:, :, :20], table, torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
        results.append([t[-8:].clone() for t in cache] + list(binding.kv_fp8_read(cache, table, lens, 470)) +
                       [t for rows in (0, 16, 128) for t in binding.attn_kv_fp8(q, cache, table, lens, causal=True, wg_rows=rows)])
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert same(a, b)
    assert torch.isfinite(results[0][-2]).all()


def test_numbers_beyond_32_bits_are_refused():
    """No number is cut to its lower half."""
    import torch
    from paper_2604_18616_amd import binding
    layer = Layer(7, 1, 4, 2, 64, 16, 64)
    q, n = torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    far = (1 << 32) + 5
    for _ in modes():
        for kw in (dict(window=far), dict(sinks=far), dict(max_len=far), dict(window=-far), dict(wg_rows=(1 << 32) + 16)):
            with pytest.raises(ValueError, match="32 bits"):
                binding.attn_kv_fp8(q, layer.cache, layer.tab, n, **kw)
        for S, first in ((far, 0), (4, far)):
            with pytest.raises(ValueError, match="32 bits"):
                binding.kv_fp8_read(layer.cache, layer.tab, n, S, first=first)
        for kw in (dict(window=2.5), dict(sinks="4")):
            with pytest.raises(TypeError):
                binding.attn_kv_fp8(q, layer.cache, layer.tab, n, **kw)
